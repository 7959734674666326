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
__host__ __device__ __forceinline__ bool sequence_fits(const Attention &a, int len, int nq, int q0)
{
    return q0 >= 0 && nq >= 0 && nq <= a.max_q && (int64_t)q0 + nq <= a.n_queries && len >= nq &&
           len <= a.max_kv &&
           (((int64_t)len + (1 << a.c.page_shift) - 1) >> a.c.page_shift) <= a.max_pages;
}
__host__ __device__ __forceinline__ bool sequence(const Attention &a, int b, int &len, int &nq, int &q0)
{
    q0 = a.cu_q[b];
    nq = a.cu_q[b + 1] - q0;
    len = a.kv_len[b];
    const bool ok = sequence_fits(a, len, nq, q0);
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
// Parts of at most `per` steps of a sequence.
__host__ __device__ __forceinline__ int fitted_parts(int steps, int per) { return (steps + per - 1) / per; }

// Steps of a part where a part's block occupies its CU alone: a round of them is a.fit blocks, and
// one block more begins another round.  total: all steps, of each row block; blocks: row blocks;
// count(per): the parts of at most `per` steps, of all row blocks.
//
// One round: the fewest steps, to a 32nd, that leave no more parts than fit.  The parts of `per`
// steps are fewer than total / per + blocks, which bounds the search from above.
// Where the row blocks alone take more than half a round, parts that do fit may be as long as the
// sequences: then parts of a half of what each of a round's blocks would get, in as many rounds as
// that takes, if that ends sooner; each of them costs about eight steps more, for its beginning and
// for its way through memory.
template <class Count>
__host__ __device__ __forceinline__ int fitted_steps(const Attention &a, int64_t total, int64_t blocks,
                                                     Count count)
{
    const int longest = (a.max_kv - 1) / kStep + 1;
    auto bounded = [&](int64_t n, int least) { return n >= longest ? longest : n > least ? (int)n : least; };
    int per = longest;
    if (blocks < a.fit) {
        int lo = bounded(total / a.fit, a.min_steps);
        per = bounded(total / (a.fit - blocks) + 1, lo);
        if (lo >= per || count(lo) <= a.fit) {
            per = lo;
        } else {
            while (per - lo > 1 + (lo >> 5)) {
                const int mid = lo + (per - lo) / 2;
                if (count(mid) <= a.fit) per = mid;
                else lo = mid;
            }
        }
    }
    if (2 * blocks <= a.fit) return per;
    const int many = bounded(total / (2 * a.fit) + 1, 2 * a.min_steps);
    if (many >= per) return per;
    const int64_t rounds = blocks <= a.fit ? 1 : (blocks + a.fit - 1) / a.fit;
    const int64_t others = (count(many) + a.fit - 1) / a.fit;
    return others * (many + 8) < rounds * per ? many : per;
}

// 256 sequences, four a lane, their loads on the way together.  (One group of 64 after the other
// took 20 us more in 256 blocks of 256 sequences.)
struct Lanes {
    static constexpr int Groups = 4, Most = 64 * Groups;
    int steps[Groups], rbs[Groups];
    __device__ __forceinline__ void load(const Attention &a, int b0)
    {
        const int lane = threadIdx.x & 63, last = a.n_seqs - 1;
        int q0[Groups], next[Groups], len[Groups];
#pragma unroll
        for (int i = 0; i < Groups; ++i) {
            const int b = min(b0 + 64 * i + lane, last);
            q0[i] = a.cu_q[b], next[i] = a.cu_q[b + 1], len[i] = a.kv_len[b];
        }
#pragma unroll
        for (int i = 0; i < Groups; ++i) {
            const int nq = next[i] - q0[i];
            bool ok = sequence_fits(a, len[i], nq, q0[i]);
            if (!ok && a.status) *a.status = KVR_E_DOMAIN;
            ok = ok && b0 + 64 * i + lane <= last;
            steps[i] = ok ? steps_of(len[i], nq) : 0;
            rbs[i] = ok ? row_blocks_of(a, nq) : 0;
        }
    }
    // This lane's steps times row blocks, and parts.
    __device__ __forceinline__ int64_t total() const
    {
        int64_t n = 0;
#pragma unroll
        for (int i = 0; i < Groups; ++i) n += (int64_t)steps[i] * rbs[i];
        return n;
    }
    __device__ __forceinline__ int64_t parts(int per) const
    {
        int64_t n = 0;
#pragma unroll
        for (int i = 0; i < Groups; ++i) n += (int64_t)fitted_parts(steps[i], per) * rbs[i];
        return n;
    }
};

// first: the first 64 sequences.
__device__ __forceinline__ int part_steps(const Attention &a, const Lane &first)
{
    if (!a.fit) {
        int64_t total = wave_total((int64_t)first.steps * first.rbs);
        for (int b0 = 64; b0 < a.n_seqs; b0 += 64) {
            const Lane x = lane_sequence(a, b0);
            total += wave_total((int64_t)x.steps * x.rbs);
        }
        return part_size(a, total);
    }
    const int longest = (a.max_kv - 1) / kStep + 1;
    if (a.n_seqs <= 64) {
        auto count = [&](int per) { return wave_total((int64_t)fitted_parts(first.steps, per) * first.rbs); };
        return fitted_steps(a, wave_total((int64_t)first.steps * first.rbs), count(longest), count);
    }
    Lanes all;
    int64_t total = 0, blocks = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += Lanes::Most) {
        all.load(a, b0);
        total += all.total();
        blocks += all.parts(longest);
    }
    auto count = [&](int per) {
        int64_t n = 0;
        if (a.n_seqs <= Lanes::Most) {
            n = all.parts(per);
        } else {
            for (int b0 = 0; b0 < a.n_seqs; b0 += Lanes::Most) {
                all.load(a, b0);
                n += all.parts(per);
            }
        }
        return wave_total(n);
    };
    return fitted_steps(a, wave_total(total), wave_total(blocks), count);
}

// Parts of a sequence: the nearest whole number (always rounding up would cut 880 row
// blocks of 31 steps into twice as many, which end in two uneven waves).
__host__ __device__ __forceinline__ int parts_of(int steps, int per)
{
    const int n = (int)((steps + (per >> 1)) / per);
    return n > 0 ? n : steps > 0;
}
__host__ __device__ __forceinline__ int parts_of(const Attention &a, int steps, int per)
{
    return a.fit ? fitted_parts(steps, per) : parts_of(steps, per);
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
