// How the sequences of an attention call are cut into parts along their cached
// tokens: from the lengths, on the device, the same in every wave.
#pragma once

#include "kvr_kv_device.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;

// ---- which part of which sequence a block works on ------------------------------

struct Part {
    int b;            // sequence; -1: nothing to do
    int part, parts;  // which of how many
    int rb;           // block of rows
    int first, last;  // steps [first, last)
    int len, nq, q0;  // cached tokens, new tokens, first query
};

__device__ __forceinline__ int wave_sum(int x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ int wave_scan(int x)   // inclusive
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if ((int)(threadIdx.x & 63) >= o) x += y;
    }
    return x;
}

__device__ __forceinline__ int lane_value(int x, int lane)   // uniform
{
    return __builtin_amdgcn_readlane(x, lane);
}

// Tokens, new tokens and first query of sequence b; false where they do not fit the call.
__device__ __forceinline__ bool sequence(const Attention &a, int b, int &len, int &nq, int &q0)
{
    q0 = a.cu_q[b];
    nq = a.cu_q[b + 1] - q0;
    len = a.kv_len[b];
    const bool ok = q0 >= 0 && nq >= 0 && nq <= a.max_q && (int64_t)q0 + nq <= a.n_queries &&
                    len >= nq && len <= a.max_kv &&
                    (((int64_t)len + (1 << a.c.page_shift) - 1) >> a.c.page_shift) <= a.max_pages;
    if (!ok) {
        if (a.status) *a.status = KVR_E_DOMAIN;
        len = nq = 0;
    }
    return ok;
}
__device__ __forceinline__ int steps_of(int len, int nq)
{
    return nq > 0 ? (len + kStep - 1) / kStep : 0;
}
__device__ __forceinline__ int row_blocks_of(const Attention &a, int nq)
{
    return (nq * a.group + a.block_rows - 1) / a.block_rows;
}

// Steps of one part: all sequences' steps (times their row blocks) over the
// target, at least min_steps.
__device__ __forceinline__ int part_steps(const Attention &a)
{
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int len = 0, nq = 0, q0;
        if (b0 + lane < a.n_seqs) sequence(a, b0 + lane, len, nq, q0);
        // at most 2^26 steps x 2^20 row blocks of 64 sequences: summed in two halves
        const int64_t w = (int64_t)steps_of(len, nq) * row_blocks_of(a, nq);
        total += (int64_t)wave_sum((int)(w & 0xffffff)) + ((int64_t)wave_sum((int)(w >> 24)) << 24);
    }
    const int64_t n = (total + a.target - 1) / a.target;
    return (int)(n > a.min_steps ? n : a.min_steps);
}

}  // namespace
}  // namespace kv
}  // namespace kvr
