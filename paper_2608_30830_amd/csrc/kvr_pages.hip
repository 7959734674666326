// The pages of a cache: rows that branch, grow, shrink and end, the pool brought
// together, pages copied.
//
// The pool's state is one count a page and the rows of the page table; every call reads and
// writes them in place, and whatever runs at the same time inside a call touches different
// words or adds to counts, so equal states give equal results.  Free pages are ranked by
// counting: a wave looks at 64 counts at a time and keeps the free ones as the bits of a word,
// blocks count their words, and a page's rank is the sum of the counts before its block plus
// the bits before its own.  These calls are small: their launches and dependent loads bound
// them.  Copying is bound by memory.
#include <algorithm>

#include "kvr_dpp.h"
#include "kvr_pages.h"

namespace kvr {
namespace pages {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ void report(const Pool &p)
{
    if (p.status) *p.status = KVR_E_DOMAIN;
}

// Entries that a row of `len` tokens holds; -1: the length does not fit.
__device__ __forceinline__ int entries(const Pool &p, int len)
{
    const int64_t n = ((int64_t)len + (1 << p.shift) - 1) >> p.shift;
    return len < 0 || n > p.width ? -1 : (int)n;
}

__device__ __forceinline__ bool in_pool(const Pool &p, int page)
{
    return page >= 0 && page < p.n_pages;
}

// A row gives a page back.
__device__ __forceinline__ void give_back(const Pool &p, int page)
{
    if (!in_pool(p, page)) {
        report(p);
    } else if (atomicSub(p.refs + page, 1) <= 0) {
        atomicAdd(p.refs + page, 1);
        report(p);
    }
}

// Sum over a block, the same in every thread.
__device__ __forceinline__ int64_t block_total(int64_t x, int64_t *lds)
{
    x = wave_total(x);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    int64_t sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += lds[w];
    __syncthreads();
    return sum;
}

// ---- branches -----------------------------------------------------------------------

// A block has one row.
__global__ __launch_bounds__(kThreads) void fork_kernel(Pool p, const int32_t *parent)
{
    const int b = blockIdx.x;
    const int a = parent[b];
    if (a < 0) return;
    const int held = p.len[b];
    // (a's row is not written in this call if it has no parent itself)
    const bool fits = a < p.n_seqs && a != b && held == 0 && parent[min(a, p.n_seqs - 1)] < 0;
    const int len = fits ? p.len[a] : 0;
    const int n = fits ? entries(p, len) : -1;
    __syncthreads();   // the row's length has been read
    if (n < 0) {
        report(p);
        return;
    }
    const int32_t *from = p.table + (int64_t)a * p.stride;
    int32_t *to = p.table + (int64_t)b * p.stride;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int page = from[i];
        to[i] = page;
        if (in_pool(p, page)) atomicAdd(p.refs + page, 1);
        else report(p);
    }
    if (threadIdx.x == 0) p.len[b] = len;
}

// ---- free pages -----------------------------------------------------------------------

// The free pages of chunk c as bits, and their number.
__device__ __forceinline__ void count_chunk(const Pool &p, int c, uint64_t *free, int32_t *count,
                                            int64_t *lds)
{
    constexpr int Words = kChunkWords / kWaves;   // of a wave
    const int lane = threadIdx.x & 63, word = (threadIdx.x >> 6) * Words;
    int sum = 0;
#pragma unroll 8
    for (int i = 0; i < Words; ++i) {
        const int64_t page = (int64_t)c * kChunk + (word + i) * 64 + lane;
        const uint64_t bits = __ballot(page < p.n_pages && p.refs[page < p.n_pages ? page : 0] <= 0);
        if (lane == 0) free[(int64_t)c * kChunkWords + word + i] = bits;
        sum += __popcll(bits);
    }
    const int64_t total = block_total(lane == 0 ? sum : 0, lds);
    if (threadIdx.x == 0) count[c] = (int)total;
}

// Free pages before chunk c, and of all chunks.
__device__ __forceinline__ void free_before(const int32_t *count, int chunks, int c, int64_t &before,
                                            int64_t &all, int64_t *lds)
{
    int64_t x = 0, y = 0;
    for (int i = threadIdx.x; i < chunks; i += kThreads) {
        const int n = count[i];
        y += n;
        if (i < c) x += n;
    }
    before = block_total(x, lds);
    all = block_total(y, lds);
}

// Calls f(page, free, its rank among the free) for the pages of chunk c, of which `before` free
// ones come before.
template <class F>
__device__ __forceinline__ void rank_chunk(const uint64_t *free, int c, int64_t before, int64_t n_pages, F f)
{
    constexpr int Words = kChunkWords / kWaves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // words of the chunk two a lane: their bits before each
    const uint64_t *w = free + (int64_t)c * kChunkWords;
    const int a = __popcll(w[2 * lane]), b = __popcll(w[2 * lane + 1]);
    const int upto = wave_incl_scan(a + b);
    for (int i = 0; i < Words; ++i) {
        const int word = wave * Words + i, l = word >> 1;
        const int first = __builtin_amdgcn_readlane(upto - (a + b), l) +
                          ((word & 1) ? __builtin_amdgcn_readlane(a, l) : 0);
        const uint64_t bits = w[word];
        const int64_t page = (int64_t)c * kChunk + word * 64 + lane;
        if (page < n_pages)
            f(page, (bits >> lane & 1) != 0, before + first + __popcll(bits & ((1ull << lane) - 1)));
    }
}

// ---- new lengths ------------------------------------------------------------------------

enum { kLeave = 0, kBack = 1, kGrow = 2, kGrowOwn = 3, kBad = 4 };

// The last block plans the rows, the others count free pages.
__global__ __launch_bounds__(kThreads) void resize_plan_kernel(Resize r)
{
    __shared__ int64_t lds[kWaves];
    const Pool &p = r.p;
    if ((int)blockIdx.x > 0) {
        count_chunk(p, blockIdx.x - 1, r.free, r.count, lds);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t base = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        Row x{};
        if (b < p.n_seqs) {
            const int want = r.new_len[b];
            if (want >= 0) {
                const int len = p.len[b];
                const int have = entries(p, len), need = entries(p, want);
                x.need = need;
                x.first = have;
                if (have < 0 || need < 0) {
                    x.mode = kBad;
                } else if (want <= len) {
                    x.mode = want < len ? kBack : kLeave;
                } else {
                    x.mode = kGrow;
                    x.take = need - have;
                    if (len & ((1 << p.shift) - 1)) {   // into a page that others hold too?
                        const int last = p.table[(int64_t)b * p.stride + have - 1];
                        if (!in_pool(p, last)) {
                            x.mode = kBad;
                            x.take = 0;
                        } else if (p.refs[last] > 1) {
                            x.mode = kGrowOwn;
                            x.take += 1;
                            x.first -= 1;
                        }
                    }
                }
            }
        }
        const int64_t upto = wave_incl_scan((int64_t)x.take);
        if (lane == 63) lds[wave] = upto;
        __syncthreads();
        int64_t before = base;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? lds[w] : 0;
            base += lds[w];
        }
        __syncthreads();
        x.start = before + upto - x.take;
        if (b < p.n_seqs) r.rows[b] = x;
    }
}

// The first blocks hand out the free pages of a chunk each, the others finish four rows each.
__global__ __launch_bounds__(kThreads) void resize_apply_kernel(Resize r)
{
    __shared__ int64_t lds[kWaves];
    const Pool &p = r.p;
    const int c = blockIdx.x;
    int64_t before, all;
    free_before(r.count, p.chunks, c, before, all, lds);
    if (c < p.chunks) {
        const Row tail = r.rows[p.n_seqs - 1];
        const int64_t taken = tail.start + tail.take;
        if (before >= taken) return;
        rank_chunk(r.free, c, before, p.n_pages, [&](int64_t page, bool free, int64_t rank) {
            if (!free || rank >= taken) return;
            int lo = 0, hi = p.n_seqs;   // the last row that starts at or before the rank
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (r.rows[mid].start <= rank) lo = mid;
                else hi = mid;
            }
            const Row x = r.rows[lo];
            if (x.start + x.take > all) return;   // it does not fit
            int32_t *entry = p.table + (int64_t)lo * p.stride + x.first + (rank - x.start);
            if (x.mode == kGrowOwn && rank == x.start) {
                const int old = *entry;
                r.copies[2 * (int64_t)lo] = old;
                r.copies[2 * (int64_t)lo + 1] = (int)page;
                give_back(p, old);
            }
            *entry = (int)page;
            p.refs[page] = 1;
        });
        return;
    }
    const int b = (c - p.chunks) * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= p.n_seqs) return;
    const Row x = r.rows[b];
    const bool grows = (x.mode == kGrow || x.mode == kGrowOwn) && (x.take == 0 || x.start + x.take <= all);
    if (x.mode == kBad || (x.mode >= kGrow && !grows)) report(p);
    if (lane == 0) {
        if (!(grows && x.mode == kGrowOwn)) r.copies[2 * (int64_t)b] = r.copies[2 * (int64_t)b + 1] = -1;
        if (grows || x.mode == kBack) p.len[b] = r.new_len[b];
    }
    if (x.mode == kBack) {
        int32_t *row = p.table + (int64_t)b * p.stride;
        for (int i = x.need + lane; i < x.first; i += 64) {
            give_back(p, row[i]);
            row[i] = -1;
        }
    }
}

// ---- compaction -----------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void count_kernel(Compact c)
{
    __shared__ int64_t lds[kWaves];
    count_chunk(c.p, blockIdx.x, c.free, c.count, lds);
}

// With U pages in use, the k-th lowest hole below U takes the k-th highest page in use, which
// lies at or beyond U: there are as many of one as of the other.
__global__ __launch_bounds__(kThreads) void pair_kernel(Compact c)
{
    __shared__ int64_t lds[kWaves];
    const Pool &p = c.p;
    int64_t before, all, holes, same;
    free_before(c.count, p.chunks, blockIdx.x, before, all, lds);
    const int64_t used = p.n_pages - all;
    // holes below U: in whole chunks, and in the words of U's own
    free_before(c.count, p.chunks, (int)(used / kChunk), holes, same, lds);
    if (used < p.n_pages) {
        const int64_t first = used / kChunk * kChunkWords, last = used / 64;   // words
        int64_t n = 0;
        for (int64_t w = first + threadIdx.x; w <= last; w += kThreads) {
            const uint64_t bits = c.free[w];
            n += __popcll(w < last ? bits : bits & ((1ull << (used & 63)) - 1));
        }
        holes += block_total(n, lds);
    }
    const int64_t limit = min(holes, c.max_moves);
    if (blockIdx.x == 0 && threadIdx.x == 0) *c.used = (int)used;
    rank_chunk(c.free, blockIdx.x, before, p.n_pages, [&](int64_t page, bool free, int64_t rank) {
        if (page >= limit && page < c.max_moves) c.moves[2 * page] = c.moves[2 * page + 1] = -1;
        if (page < used) {
            if (free && rank < limit) c.moves[2 * rank + 1] = (int)page;
            return;
        }
        const int64_t k = used - 1 - (page - rank);   // among those in use, from the highest
        const bool moves = !free && k < limit;
        if (moves) c.moves[2 * k] = (int)page;
        c.where[page] = moves ? (int)k : -1;
    });
}

// The first blocks carry the counts over, the others change four rows of the table each.
__global__ __launch_bounds__(kThreads) void move_kernel(Compact c, int move_blocks)
{
    const Pool &p = c.p;
    if ((int)blockIdx.x < move_blocks) {
        const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
        if (k >= c.max_moves) return;
        const int from = c.moves[2 * k], to = c.moves[2 * k + 1];
        if (from < 0) return;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
        return;
    }
    const int b = (blockIdx.x - move_blocks) * kWaves + (threadIdx.x >> 6);
    if (b >= p.n_seqs) return;
    const int n = entries(p, p.len[b]), used = *c.used;
    if (n < 0) report(p);
    int32_t *row = p.table + (int64_t)b * p.stride;
    for (int i = threadIdx.x & 63; i < n; i += 64) {
        const int page = row[i];
        if (!in_pool(p, page)) {
            report(p);
        } else if (page >= used) {
            const int k = c.where[page];
            if (k >= 0) row[i] = c.moves[2 * (int64_t)k + 1];
        }
    }
}

// ---- copies ---------------------------------------------------------------------------

// A block has one of `split` shares of a page of one tensor; W bytes a thread at a time, four
// in flight.
template <class T, bool Whole>
__global__ __launch_bounds__(kThreads) void copy_kernel(Copy c)
{
    constexpr int W = sizeof(T), U = 4;
    const int64_t block = (int64_t)blockIdx.z * kv::kMaxGrid + blockIdx.x;
    const int64_t pair = block / c.split;
    if (pair >= c.n_pairs) return;
    const int share = (int)(block - pair * c.split);
    const int from = c.pairs[2 * pair], to = c.pairs[2 * pair + 1];
    if (from < 0 || to < 0) return;
    if (from >= c.n_pages || to >= c.n_pages) {
        if (c.status) *c.status = KVR_E_DOMAIN;
        return;
    }
    char *data = c.data[blockIdx.y];
    const char *src = data + from * c.page_stride;
    char *dst = data + to * c.page_stride;
    const int64_t run = c.run / W, units = run * c.inner * c.outer;
    const int64_t per = (units + c.split - 1) / c.split;
    const int64_t end = min(units, per * (share + 1));
    auto at = [&](int64_t u) {
        if (Whole) return u * W;
        const int64_t r = u / run, o = r / c.inner;
        return o * c.outer_stride + (r - o * c.inner) * c.inner_stride + (u - r * run) * W;
    };
    for (int64_t u = per * share + threadIdx.x; u < end; u += kThreads * U) {
        T x[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (u + i * kThreads < end) x[i] = *reinterpret_cast<const T *>(src + at(u + i * kThreads));
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (u + i * kThreads < end) *reinterpret_cast<T *>(dst + at(u + i * kThreads)) = x[i];
    }
}

template <class T>
hipError_t copy_width(const Copy &c, dim3 grid, hipStream_t stream)
{
    if (c.outer == 1 && c.inner == 1) copy_kernel<T, true><<<grid, kThreads, 0, stream>>>(c);
    else copy_kernel<T, false><<<grid, kThreads, 0, stream>>>(c);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fork(const Pool &p, const int32_t *parent, hipStream_t stream)
{
    fork_kernel<<<p.n_seqs, kThreads, 0, stream>>>(p, parent);
    return hipGetLastError();
}

hipError_t launch_resize(const Resize &r, hipStream_t stream)
{
    resize_plan_kernel<<<r.p.chunks + 1, kThreads, 0, stream>>>(r);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    resize_apply_kernel<<<r.p.chunks + (unsigned)kv::cdiv(r.p.n_seqs, kWaves), kThreads, 0, stream>>>(r);
    return hipGetLastError();
}

hipError_t launch_compact(const Compact &c, hipStream_t stream)
{
    count_kernel<<<c.p.chunks, kThreads, 0, stream>>>(c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    pair_kernel<<<c.p.chunks, kThreads, 0, stream>>>(c);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int moves = (int)kv::cdiv(c.max_moves, kThreads);
    const unsigned rows = (unsigned)kv::cdiv(c.p.n_seqs, kWaves);
    if (moves + rows == 0) return hipSuccess;
    move_kernel<<<moves + rows, kThreads, 0, stream>>>(c, moves);
    return hipGetLastError();
}

hipError_t launch_copy(const Copy &c, hipStream_t stream)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const dim3 grid = kv::grid_of(c.n_pairs * c.split, c.n_buffers);
    switch (c.width) {
    case 16: return copy_width<u32x4>(c, grid, stream);
    case 4: return copy_width<uint32_t>(c, grid, stream);
    default: return copy_width<uint8_t>(c, grid, stream);
    }
}

}  // namespace pages
}  // namespace kvr
