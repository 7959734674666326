// The pages of a cache: rows that branch, grow, shrink and end, the pool brought
// together, pages copied.
//
// The pool's state is one count a page and the rows of the page table; every call reads and
// writes them in place, and whatever runs at the same time inside a call touches different
// words or adds to counts, so equal states give equal results.  Free pages are ranked by
// counting: a wave looks at 64 counts at a time and keeps the free ones as the bits of a word,
// blocks count their words, and a page's rank is the sum of the counts before its block plus
// the bits before its own.  These calls are small: their launches and dependent loads bound
// them.  In 4,096 pages a call in a graph takes 2 us (a branch), 7 us (new lengths of 64 rows) and 7 us
// (compaction, 64 rows).  Copying is bound by memory: 1.24 GB, read and written, in 240 us (5.2 TB/s).
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

// A row gives a page back that it held when the call began.
__device__ __forceinline__ void give_back(const Pool &p, int page)
{
    if (atomicSub(p.refs + page, 1) <= 0) {
        atomicAdd(p.refs + page, 1);
        report(p);
    }
}
// Up to four entries, which become -1: the atomics of one wait together.  free: the pages that were
// free when the call began, as bits.  What names one of them is reported, whether or not another row
// has taken the page meanwhile, whose count it would lower.  (A load before each atomic: 64 rows in
// 4,096 pages 7.1 us a call without it, 7.3 with it; one row of 6,144 pages 28.6 and 32.7.)
__device__ __forceinline__ void give_back(const Pool &p, const uint64_t *free, int32_t *const (&at)[4])
{
    int page[4], held[4];
    bool counts[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) page[k] = at[k] ? *at[k] : -1;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        counts[k] = in_pool(p, page[k]) && !(free[page[k] >> 6] >> (page[k] & 63) & 1);
#pragma unroll
    for (int k = 0; k < 4; ++k) held[k] = counts[k] ? atomicSub(p.refs + page[k], 1) : 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (!at[k]) continue;
        if (held[k] <= 0) {   // outside the pool, free, or given back more often than held
            if (counts[k]) atomicAdd(p.refs + page[k], 1);
            report(p);
        }
        *at[k] = -1;
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

// The free pages of `words` words from the block's first one on as bits, and their number.
template <int Waves>
__device__ __forceinline__ int count_words(const Pool &p, int64_t first, int words, uint64_t *free)
{
    const int lane = threadIdx.x & 63;
    int sum = 0;
    for (int w = threadIdx.x >> 6; w < words; w += 4 * Waves) {
        int refs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // loads first
            const int64_t page = (first + w + i * Waves) * 64 + lane;
            refs[i] = w + i * Waves < words && page < p.n_pages ? p.refs[page] : 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t bits = __ballot(refs[i] <= 0);
            if (lane == 0 && w + i * Waves < words) free[w + i * Waves] = bits;
            sum += __popcll(bits);
        }
    }
    return lane == 0 ? sum : 0;
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

// The pages of `words` words from the block's first one on, of which `before` free ones come
// before: f(page, free, rank among the free).  Each wave counts the words before its own.
template <int Waves, class F>
__device__ __forceinline__ void rank_words(const Pool &p, const uint64_t *free, int64_t first, int words,
                                           int64_t before, F f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (words + Waves - 1) / Waves, w0 = wave * per, w1 = min(w0 + per, words);
    int64_t x = 0;
    for (int w = lane; w < w0; w += 64) x += __popcll(free[w]);
    int64_t rank = before + wave_total(x);
    for (int w = w0; w < w1; ++w) {
        const uint64_t bits = free[w];
        const int64_t page = (first + w) * 64 + lane;
        if (page < p.n_pages) f(page, (bits >> lane & 1) != 0, rank + __popcll(bits & ((1ull << lane) - 1)));
        rank += __popcll(bits);
    }
}

// ---- new lengths ------------------------------------------------------------------------

enum { kLeave = 0, kBack = 1, kGrow = 2, kGrowOwn = 3, kBad = 4 };

// What row b does, but for its start.
__device__ __forceinline__ Row plan_row(const Resize &r, int b)
{
    const Pool &p = r.p;
    Row x{};
    const int want = r.new_len[b], len = p.len[b];
    if (want < 0) return x;
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
    return x;
}

// Page `page`, free and of this rank, goes to row b.
__device__ __forceinline__ void give(const Resize &r, int b, const Row &x, int64_t page, int64_t rank)
{
    const Pool &p = r.p;
    int32_t *entry = p.table + (int64_t)b * p.stride + x.first + (rank - x.start);
    if (x.mode == kGrowOwn && rank == x.start) {
        const int old = *entry;
        r.copies[2 * (int64_t)b] = old;
        r.copies[2 * (int64_t)b + 1] = (int)page;
        give_back(p, old);
    }
    *entry = (int)page;
    p.refs[page] = 1;
}

// Row b's length, and its pages to copy if there are none; all: the pages that are free.
__device__ __forceinline__ void end_row(const Resize &r, int b, const Row &x, int64_t all)
{
    const bool grows = (x.mode == kGrow || x.mode == kGrowOwn) && (x.take == 0 || x.start + x.take <= all);
    if (x.mode == kBad || (x.mode >= kGrow && !grows)) report(r.p);
    if (!(grows && x.mode == kGrowOwn)) r.copies[2 * (int64_t)b] = r.copies[2 * (int64_t)b + 1] = -1;
    if (grows || x.mode == kBack) r.p.len[b] = r.new_len[b];
}
// The rest of what row b does, by one wave.
__device__ __forceinline__ void finish_row(const Resize &r, int b, const Row &x, int64_t all)
{
    const Pool &p = r.p;
    const int lane = threadIdx.x & 63;
    if (lane == 0) end_row(r, b, x, all);
    if (x.mode == kBack) {
        int32_t *row = p.table + (int64_t)b * p.stride;
        for (int i = x.need + lane; i < x.first; i += 4 * 64) {
            int32_t *at[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) at[k] = i + k * 64 < x.first ? row + i + k * 64 : nullptr;
            give_back(p, r.free, at);
        }
    }
}

// The last row that starts at or before a rank.
template <class Start>
__device__ __forceinline__ int row_of_rank(int n_seqs, int64_t rank, Start start)
{
    int lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start(mid) <= rank) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The first block plans the rows, the others count free pages.
__global__ __launch_bounds__(kThreads) void resize_plan_kernel(Resize r)
{
    __shared__ int64_t lds[kWaves];
    const Pool &p = r.p;
    if ((int)blockIdx.x > 0) {
        const int c = blockIdx.x - 1;
        const int64_t n = block_total(count_words<kWaves>(p, (int64_t)c * p.words, p.words, r.free + (int64_t)c * p.words), lds);
        if (threadIdx.x == 0) r.count[c] = (int)n;
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t base = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        Row x{};
        if (b < p.n_seqs) x = plan_row(r, b);
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
        rank_words<kWaves>(p, r.free + (int64_t)c * p.words, (int64_t)c * p.words, p.words, before,
                           [&](int64_t page, bool free, int64_t rank) {
            if (!free || rank >= taken) return;
            const int b = row_of_rank(p.n_seqs, rank, [&](int i) { return r.rows[i].start; });
            const Row x = r.rows[b];
            if (x.start + x.take <= all) give(r, b, x, page, rank);
        });
        return;
    }
    const int b = (c - p.chunks) * kWaves + (threadIdx.x >> 6);
    if (b < p.n_seqs) finish_row(r, b, r.rows[b], all);
}

// The same for a small pool, by one block, rows in LDS.  (The counts of free pages are taken before
// any changes.)  What rows give back is spread over all threads, four entries each at a time: the
// atomics of one wait together.
constexpr int kWide = 1024, kWideWaves = kWide / 64;

// Exclusive sum over the block's threads; total: of all.  lds: [kWideWaves].
__device__ __forceinline__ int64_t wide_scan(int64_t x, int64_t *lds, int64_t &total)
{
    const int64_t upto = wave_incl_scan(x);
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = upto;
    __syncthreads();
    int64_t before = upto - x;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += lds[w];
        total += lds[w];
    }
    __syncthreads();
    return before;
}

__global__ __launch_bounds__(kWide) void resize_small_kernel(Resize r)
{
    __shared__ uint64_t free[kSmallResize / 64];
    __shared__ Row rows[kSmallSeqs];
    __shared__ int32_t back[kSmallSeqs];   // entries that the rows before give back
    __shared__ int64_t sums[kWideWaves];
    const Pool &p = r.p;
    const int lane = threadIdx.x & 63;
    const int words = (int)((p.n_pages + 63) >> 6);
    const int mine = wave_total(count_words<kWideWaves>(p, 0, words, free));
    const int b = threadIdx.x;   // at most kWide rows
    Row x{};
    if (b < p.n_seqs) x = plan_row(r, b);
    int64_t all, taken, returned;
    wide_scan(lane == 0 ? mine : 0, sums, all);
    x.start = wide_scan(x.take, sums, taken);
    back[b] = (int32_t)wide_scan(x.mode == kBack ? x.first - x.need : 0, sums, returned);
    rows[b] = x;
    __syncthreads();
    rank_words<kWideWaves>(p, free, 0, words, 0, [&](int64_t page, bool is_free, int64_t rank) {
        if (!is_free || rank >= taken) return;
        const int to = row_of_rank(p.n_seqs, rank, [&](int i) { return rows[i].start; });
        const Row y = rows[to];
        if (y.start + y.take <= all) give(r, to, y, page, rank);
    });
    for (int i0 = threadIdx.x; i0 < returned; i0 += 4 * kWide) {
        int32_t *at[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * kWide;
            at[k] = nullptr;
            if (i >= returned) continue;
            const int of = row_of_rank(p.n_seqs, i, [&](int j) { return (int64_t)back[j]; });
            at[k] = p.table + (int64_t)of * p.stride + rows[of].need + (i - back[of]);
        }
        give_back(p, free, at);
    }
    if (b < p.n_seqs) end_row(r, b, x, all);
}

// ---- compaction -----------------------------------------------------------------------

// With U pages in use, the k-th lowest hole below U takes the k-th highest page in use, which
// lies at or beyond U: there are as many of one as of the other.
__device__ __forceinline__ void pair_page(const Compact &c, int64_t page, bool free, int64_t rank, int64_t used,
                                          int64_t limit)
{
    if (page >= limit && page < c.max_moves) c.moves[2 * page] = c.moves[2 * page + 1] = -1;
    if (page < used) {
        if (free && rank < limit) c.moves[2 * rank + 1] = (int)page;
        return;
    }
    const int64_t k = used - 1 - (page - rank);   // among those in use, from the highest
    const bool moves = !free && k < limit;
    if (moves) c.moves[2 * k] = (int)page;
    c.where[page] = moves ? (int)k : -1;
}
// Free pages before `used` among words from `first` on that begin before it.
__device__ __forceinline__ int64_t holes_of(const uint64_t *free, int64_t first, int64_t used, int threads)
{
    int64_t n = 0;
    for (int64_t w = first + threadIdx.x; w * 64 < used; w += threads)
        n += __popcll((w + 1) * 64 <= used ? free[w] : free[w] & ((1ull << (used & 63)) - 1));
    return n;
}
__device__ __forceinline__ void move_counts(const Compact &c, int64_t k)
{
    const int from = c.moves[2 * k], to = c.moves[2 * k + 1];
    if (from < 0) return;
    c.p.refs[to] = c.p.refs[from];
    c.p.refs[from] = 0;
}
// One wave changes row b of the table.
__device__ __forceinline__ void move_row(const Compact &c, int b, int used)
{
    const Pool &p = c.p;
    const int n = entries(p, p.len[b]);
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

__global__ __launch_bounds__(kThreads) void count_kernel(Compact c)
{
    __shared__ int64_t lds[kWaves];
    const int64_t first = (int64_t)blockIdx.x * c.p.words;
    const int64_t n = block_total(count_words<kWaves>(c.p, first, c.p.words, c.free + first), lds);
    if (threadIdx.x == 0) c.count[blockIdx.x] = (int)n;
}

__global__ __launch_bounds__(kThreads) void pair_kernel(Compact c)
{
    __shared__ int64_t lds[kWaves];
    const Pool &p = c.p;
    int64_t before, all, holes, same;
    free_before(c.count, p.chunks, blockIdx.x, before, all, lds);
    const int64_t used = p.n_pages - all, chunk = used / (64 * (int64_t)p.words);
    // holes below U: in whole chunks, and in the words of U's own
    free_before(c.count, p.chunks, (int)chunk, holes, same, lds);
    holes += block_total(holes_of(c.free, chunk * p.words, used, kThreads), lds);
    if (blockIdx.x == 0 && threadIdx.x == 0) *c.used = (int)used;
    const int64_t first = (int64_t)blockIdx.x * p.words, limit = min(holes, c.max_moves);
    rank_words<kWaves>(p, c.free + first, first, p.words, before,
                       [&](int64_t page, bool free, int64_t rank) { pair_page(c, page, free, rank, used, limit); });
}

// The first blocks carry the counts over, the others change four rows of the table each.
__global__ __launch_bounds__(kThreads) void move_kernel(Compact c, int move_blocks)
{
    if ((int)blockIdx.x < move_blocks) {
        const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
        if (k < c.max_moves) move_counts(c, k);
        return;
    }
    const int b = (blockIdx.x - move_blocks) * kWaves + (threadIdx.x >> 6);
    if (b < c.p.n_seqs) move_row(c, b, *c.used);
}

// The same for a small pool, by one block.
__global__ __launch_bounds__(kWide) void compact_small_kernel(Compact c)
{
    __shared__ uint64_t free[kSmallCompact / 64];
    __shared__ int part[kWideWaves], hole[kWideWaves];
    const Pool &p = c.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int words = (int)((p.n_pages + 63) >> 6);
    const int mine = wave_total(count_words<kWideWaves>(p, 0, words, free));
    if (lane == 0) part[wave] = mine;
    __syncthreads();
    int64_t used = p.n_pages;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) used -= part[w];
    const int64_t holes = wave_total(holes_of(free, 0, used, kWide));
    if (lane == 0) hole[wave] = (int)holes;
    __syncthreads();
    int64_t limit = 0;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) limit += hole[w];
    limit = min(limit, c.max_moves);
    if (threadIdx.x == 0) *c.used = (int)used;
    rank_words<kWideWaves>(p, free, 0, words, 0,
                           [&](int64_t page, bool is_free, int64_t rank) { pair_page(c, page, is_free, rank, used, limit); });
    __syncthreads();   // moves and `where` are complete
    for (int64_t k = threadIdx.x; k < limit; k += kWide) move_counts(c, k);
    for (int b = wave; b < p.n_seqs; b += kWideWaves) move_row(c, b, (int)used);
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
    const int64_t entries = (int64_t)r.p.n_seqs * r.p.width;
    if (r.p.n_pages <= kSmallResize && r.p.n_seqs <= kSmallSeqs && entries <= kSmallEntries) {
        resize_small_kernel<<<1, kWide, 0, stream>>>(r);
        return hipGetLastError();
    }
    resize_plan_kernel<<<r.p.chunks + 1, kThreads, 0, stream>>>(r);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    resize_apply_kernel<<<r.p.chunks + (unsigned)kv::cdiv(r.p.n_seqs, kWaves), kThreads, 0, stream>>>(r);
    return hipGetLastError();
}

hipError_t launch_compact(const Compact &c, hipStream_t stream)
{
    const int64_t entries = (int64_t)c.p.n_seqs * c.p.width;
    if (c.p.n_pages <= kSmallCompact && c.p.n_seqs <= kFewSeqs && entries <= kSmallEntries) {
        compact_small_kernel<<<1, kWide, 0, stream>>>(c);
        return hipGetLastError();
    }
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
