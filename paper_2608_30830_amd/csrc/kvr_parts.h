// How the sequences of an attention call are cut into parts along their cached
// tokens: from the lengths, on the device, the same in every wave.  The arithmetic is
// for the host too, so that it can be checked there.
#pragma once

#include "kvr_dpp.h"
#include "kvr_kv_device.h"

namespace kvr {
namespace kv {
namespace {

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

__device__ __forceinline__ int lane_value(int x, int lane)   // uniform
{
    return __builtin_amdgcn_readlane(x, lane);
}

// Tokens, new tokens and first query of sequence b; false where they do not fit the call.
__host__ __device__ __forceinline__ bool sequence(const Attention &a, int b, int &len, int &nq, int &q0)
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
__host__ __device__ __forceinline__ int steps_of(int len, int nq)
{
    return nq > 0 ? (len + kStep - 1) / kStep : 0;
}
__host__ __device__ __forceinline__ int row_blocks_of(const Attention &a, int nq)
{
    return (nq * a.group + a.block_rows - 1) / a.block_rows;
}

// 64 sequences, one a lane.
struct Lane {
    int len, nq, q0, steps, rbs;
};
__device__ __forceinline__ Lane lane_sequence(const Attention &a, int b0)
{
    Lane x{};
    const int b = b0 + (threadIdx.x & 63);
    if (b < a.n_seqs) sequence(a, b, x.len, x.nq, x.q0);
    x.steps = steps_of(x.len, x.nq);
    x.rbs = row_blocks_of(a, x.nq);
    return x;
}

// Steps of one part, from the total of all sequences' steps times their row blocks: the
// total over the target, at least min_steps.
__host__ __device__ __forceinline__ int part_size(const Attention &a, int64_t total)
{
    // A total is at most 2^12 sequences x 2^25 steps x 2^18 row blocks.  Parts longer than the
    // longest sequence are no fewer, so the quotient is cut there, before it becomes an int.
    const int longest = (a.max_kv - 1) / kStep + 1;
    const double n = floor((double)total / (double)a.target) + 1.0;
    const int per = n < (double)longest ? (int)n : longest;
    return per > a.min_steps ? per : a.min_steps;
}
// first: the first 64 sequences.
__device__ __forceinline__ int part_steps(const Attention &a, const Lane &first)
{
    int64_t total = wave_total((int64_t)first.steps * first.rbs);
    for (int b0 = 64; b0 < a.n_seqs; b0 += 64) {
        const Lane x = lane_sequence(a, b0);
        total += wave_total((int64_t)x.steps * x.rbs);
    }
    return part_size(a, total);
}

// Parts of a sequence: the nearest whole number (always rounding up would cut 880 row
// blocks of 31 steps into twice as many, which end in two uneven waves).
__host__ __device__ __forceinline__ int parts_of(int steps, int per)
{
    const int n = (int)((steps + (per >> 1)) / per);
    return n > 0 ? n : steps > 0;
}

// Whether the items of a sequence, which begin at item `base`, are all among the planned
// ones: launched, and with room in the workspace.  The plan counts on sequences that
// follow one another in the queries; where cu_q decreases (one sequence then has fewer than
// no tokens and is reported), the others may have the same queries several times.
__host__ __device__ __forceinline__ bool planned(const Attention &a, int64_t base, int parts,
                                                 int row_blocks)
{
    return base + (int64_t)parts * row_blocks <= a.max_items;
}

}  // namespace
}  // namespace kv
}  // namespace kvr
