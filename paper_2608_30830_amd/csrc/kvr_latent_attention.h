// Attention over the latent cache (the absorbed form):
//   out_r = sum_j p_rj x_j[: rank] / sum_j p_rj,   p_rj = exp(scale q_r . x_j - m_r),
// one pass over the cached rows x_j with the running maximum m_r and sum.  A row r is one head
// of one new token; all of them share the cached rows.
//
// Matrix instructions (16x16x32) compute S^T = X Q^T and O^T = X[: rank]^T P^T, so that a lane
// owns one row r (lane mod 16) throughout and P^T leaves the first product in the layout that
// the second one takes.  Cached rows lie in LDS as they lie in memory, 16-byte chunks exchanged
// within a row so that neither reading disturbs the banks; the first product reads them along
// the row (256 bytes a clock), the second one across (ds_read_b64_tr_b16 turns 4x16 elements
// around, 128 bytes a clock).  So a cached row is fetched once and is key and value.  16-bit rows
// go from memory to LDS without passing through registers; codes are converted to bfloat16 on
// the way, exactly.
//
// Weights are rounded to the products' 16-bit type (bfloat16 for codes, which it holds exactly) and
// the outputs divided by the sum of the rounded weights, so that a large weight's rounding cancels;
// scores, sums and outputs are held in 32 bits.
//
// Up to 16 rows (FewRows) each of a block's four waves has all of them and takes every fourth
// step of 32 cached rows in a tile of its own: no barrier, and the other waves' loads are on their
// way while one computes.  Memory bounds this: 64 sequences of 8,192 tokens, 16 heads of 512 + 64, take 67
// us in 8 bits (4.7 TB/s, with the conversions in the way) and, with the joining, 122 in 16 bits (4.9
// TB/s; 6.3 from one length to the next).  A block needs about 5 us before its first product, and its first step, whose
// instructions are not in the cache, about 4: 1,000 tokens of one sequence take 14 us in 8 blocks.
//
// Beyond (ManyRows) the waves share tiles of 64 cached rows, one of two in LDS while the next one
// is on its way.  A block has groups of two waves, each with up to RT times 16 rows: for the scores
// they divide the cached rows, for the outputs the columns, and exchange the weights through LDS.  So each
// fragment that a wave reads meets all its rows, no wave reads the whole tile twice, and the
// accumulators of a wave are half a row wide, which leaves registers to read LDS a group of
// fragments ahead.  (Four waves of 32 rows each and no exchange: 483 us where this takes 276, 64
// sequences of 8,192 tokens and 128 heads of 512 + 64.)  Reading LDS bounds it, with the matrix
// instructions: 128 heads run at 650 TFLOP/s from one length to the next, of rank 256, where 128 rows
// share what is read, at 760.  A wave works on the tiles of 16 rows that it has, and a group has its
// second one when all have one: 144 rows of rank 256 over 131,071 tokens take 52 us in two blocks of 80 and 64,
// where two of 128 and 16 took 61.  Loads made between the products, a few at a time, were slower: each
// waits until the queue of loads has room.
//
// Each source that includes this header builds the kernels for one cache format.
#pragma once

#include "kvr_attention.h"
#include "kvr_latent.h"

namespace kvr {
namespace kv {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// The same in all lanes, as the compiler may not see.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}
// 16 bytes a lane from memory into LDS, past the registers: lane l's at `to` + 16 l; `to` and
// `base` are the same in all lanes.  In assembly, because the compiler waits for every such load
// before the next read of LDS, of whatever buffer: the loops below count them themselves (there
// are no output registers, and the compiler's own waits only become longer by them; nothing else
// here uses m0).
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(uniform((int)to)), "v"(offset), "s"(uniform((int64_t)base)) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *p, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(uniform((int)to)), "v"(p) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}
// Waits until at most N of this wave's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
// A barrier that waits for LDS, but for no load.
__device__ __forceinline__ void block_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// Whether any thread of the block says so; flag: a word of LDS that nobody else uses.
__device__ __forceinline__ bool block_any(bool x, uint32_t *flag)
{
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    if (x) *flag = 1;
    __syncthreads();
    return *flag != 0;
}

// Four elements of this lane's column (lane mod 16) of a block of four rows and 16 columns; p:
// columns 4 (lane mod 4) on of row lane / 4 mod 4.
__device__ __forceinline__ u32x2 read_across(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// Two 16-bit values added to a 32-bit sum.
template <int MT>
__device__ __forceinline__ float add_pair(uint32_t x, float sum)
{
    if (MT == KVR_DT_BF16)
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x),
                                               __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x), __builtin_bit_cast(f16x2, 0x3c003c00u), sum, false);
}

// Infinities and NaN of two 16-bit values to zero.
template <int MT>
__device__ __forceinline__ void clear_odd2(uint32_t &x)
{
    constexpr uint32_t e = MT == KVR_DT_FP16 ? 0x7c00u : 0x7f80u;
    if ((x & e) == e) x &= 0xffff0000u;
    if ((x & e << 16) == e << 16) x &= 0xffffu;
}
// Whether there are any among the values whose exponents have been combined into the halves of
// `most`.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int MT>
__device__ __forceinline__ void keep_most(uint32_t x, u16x2 &most)
{
    constexpr uint32_t e = MT == KVR_DT_FP16 ? 0x7c007c00u : 0x7f807f80u;
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x & e));
}
template <int MT>
__device__ __forceinline__ bool any_odd(u16x2 most)
{
    constexpr uint16_t e = MT == KVR_DT_FP16 ? 0x7c00 : 0x7f80;
    return __ballot(most[0] == e || most[1] == e) != 0;
}

// What the kernels share.  Rows: cached rows of a tile, Movers: waves that bring it.
template <int FMT, int RK, int RO, int TileRows, int Movers>
struct LatentTile {
    static constexpr int Rank = 32 * RK, NB = RK + RO;      // blocks of 32 elements of a row
    static constexpr bool Quant = FMT == KVR_KV_FP8;
    static constexpr int MT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // product type
    // LDS bytes: the latents of a tile, its shared keys
    static constexpr int Main = TileRows * Rank * 2, Tail = TileRows * 64 * RO, Tile = Main + Tail;
    static constexpr int Parts = TileRows / 16;             // each of them within a page

    const LatentAttention &la;
    const Attention &a;
    const int n, g, lane;
    int item, len, prefix, q0, rows;
    const int32_t *pages;
    int held, held_at;   // entries held_at on of the sequence's row of the page table, one a lane
    uint32_t key_at, tail_at, val_at;   // byte offsets of this lane in a tile

    // Chunk c of row r lies at c ^ (r mod 16) of its row (the latents), c ^ (r / 2 mod 8) or
    // c ^ (r / 4 mod 4) (the shared keys, 8 or 4 chunks): 16 rows' chunks of one column then lie
    // in 16 different places of 256 bytes.
    __device__ __forceinline__ static int tail_swizzle(int r) { return RO == 2 ? r >> 1 & 7 : r >> 2 & 3; }

    __device__ LatentTile(const LatentAttention &l)
        : la(l), a(l.a), n(threadIdx.x & 15), g((threadIdx.x & 63) >> 4), lane(threadIdx.x & 63)
    {
        key_at = n * (Rank * 2) + ((g ^ n) << 4);
        tail_at = Main + n * (64 * RO) + ((g ^ tail_swizzle(n)) << 4);
        const int r = 4 * g + (n >> 2);
        val_at = r * (Rank * 2) + (((n & 3) >> 1 ^ r) << 4) + ((n & 1) << 3);
    }
    // What this block works on.  A part's row blocks read the same cached rows: they are on one XCD
    // (blocks go to the eight in turn), at the same time, so that its cache has them for all but one.
    // (Four sequences of 32,768 tokens, 144 rows of rank 512: 87 us, with the parts' blocks in a row 90.)
    __device__ __forceinline__ Part find()
    {
        const int b = blockIdx.x, whole = la.span > 1 ? gridDim.x / (8 * la.span) * (8 * la.span) : 0;
        const int j = b >> 3;
        item = b < whole ? ((j / la.span << 3) + (b & 7)) * la.span + j % la.span : b;
        return find_part(a, item);
    }
    __device__ __forceinline__ void begin(const Part &p)
    {
        len = uniform(p.len);
        prefix = uniform(p.len - p.nq);
        q0 = uniform(p.q0);
        rows = uniform(p.nq * a.group);
        pages = a.pages + (int64_t)uniform(p.b) * a.pages_stride;
    }

    // ---- rows into LDS ---------------------------------------------------------------------

    __device__ __forceinline__ void hold(int entry)
    {
        held_at = entry;
        held = pages[min((int64_t)entry + lane, a.max_pages - 1)];
    }
    __device__ __forceinline__ int page_of(int t)
    {
        const int entry = t >> a.c.page_shift;
        if (entry < held_at || entry >= held_at + 64) hold(entry);
        int page = __builtin_amdgcn_readlane(held, entry - held_at);
        if (page < 0 || page >= a.c.n_pages) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            page = 0;
        }
        return page;
    }
    // The part whose shared keys a wave brings first (with eight waves a half of them, or as another
    // wave does).
    __device__ __forceinline__ static int tail_part(int mover)
    {
        return Movers <= Parts ? mover : RO == 2 || Quant ? mover >> 1 : mover & 3;
    }
    // Where the rows of a tile lie in the cache; rows past its last one read as that one.
    struct Where {
        int64_t at[Parts], sat[Parts];   // byte offset of each 16 rows
        int64_t mine, smine;             // of part tail_part(mover)
        int last;                        // the tile's last row
    };
    __device__ __forceinline__ Where locate(int t, int end, int mover)   // t: the first row
    {
        Where w;
        w.last = min(end - 1 - t, TileRows - 1);
        w.mine = w.smine = 0;
#pragma unroll
        for (int i = 0; i < Parts; ++i) {
            const int u = t + min(16 * i, w.last & ~15);
            const int page = page_of(u), off = u & ((1 << a.c.page_shift) - 1);
            w.at[i] = uniform(page * la.c.page_stride + off * la.c.token_stride);
            w.sat[i] = Quant ? uniform(page * la.c.spage_stride + off * la.c.stoken_stride) : 0;
            if (i == tail_part(mover)) w.mine = w.at[i], w.smine = w.sat[i];
        }
        return w;
    }
    // Row r of part i, as its number in the 16 that at[i] points to.
    __device__ __forceinline__ static int row_of(int last, int i, int r)
    {
        return 16 * i > last ? last & 15 : min(r, last - 16 * i);
    }

    // 16-bit rows: wave `mover` brings every Movers-th KB of the latents, and the shared keys of
    // parts mover, mover + Movers, ...
    static constexpr int RowChunks = Rank / 8, TailChunks = 4 * RO;        // of a row
    static constexpr int RowsMain = 64 / RowChunks, RowsTail = 64 / TailChunks;   // of a load
    static constexpr int TailOf = 16 / RowsTail;                           // loads of a part's shared keys
    static constexpr int MainOf = Main / 1024 / Movers;
    static constexpr int Loads = MainOf + (Movers <= Parts ? Parts / Movers * TailOf : 1);
    template <bool Whole>
    __device__ __forceinline__ void fetch_rows(const Where &w, int mover, uint32_t tile) const
    {
        static_assert(Movers * RowsMain <= 16 && (Parts % Movers == 0 || (Parts == 4 && Movers == 8)), "whole parts");
        const uint32_t stride = (uint32_t)la.c.token_stride;
        static_for<0, Loads>([&](auto L) {
            constexpr int l = decltype(L)::value;
            if constexpr (l < MainOf) {
                constexpr int per = RowsMain > 1 ? RowChunks : 64;
                constexpr int i = l * Movers * RowsMain / 16;
                const int j = l * Movers + mover;
                const int first = (j * RowsMain) & 15, r = first + lane / per;   // in part i
                const uint32_t c = 16 * ((lane & (RowChunks - 1)) ^ r);
                if (Whole)
                    load_to_lds(la.c.rows + w.at[i] + first * la.c.token_stride, lane / per * stride + c, tile + j * 1024);
                else load_to_lds(la.c.rows + w.at[i] + row_of(w.last, i, r) * la.c.token_stride + c, tile + j * 1024);
            } else {
                constexpr int i0 = (l - MainOf) / TailOf * Movers;
                const int k = Movers <= Parts ? (l - MainOf) % TailOf : RO == 2 ? mover & 1 : 0;
                const int i = i0 + tail_part(mover);
                const int64_t at = Movers == 1 ? w.at[i0] : w.mine;
                const int first = k * RowsTail, r = first + lane / TailChunks;
                const uint32_t c = Rank * 2 + 16 * ((lane & (TailChunks - 1)) ^ tail_swizzle(r));
                const uint32_t to = tile + Main + i * (16 * 64 * RO) + k * 1024;
                if (Whole) load_to_lds(la.c.rows + at + first * la.c.token_stride, lane / TailChunks * stride + c, to);
                else load_to_lds(la.c.rows + at + row_of(w.last, i, r) * la.c.token_stride + c, to);
            }
        });
    }
    __device__ __forceinline__ void fetch(const Where &w, int mover, uint32_t tile) const
    {
        if (w.last == TileRows - 1) fetch_rows<true>(w, mover, tile);
        else fetch_rows<false>(w, mover, tile);
    }

    // Rows of codes: 16 codes a lane, converted into two chunks.  Loads 0 to MainLoads - 1 are of
    // latents, the others of the shared keys of a part each.
    static constexpr int MainLoads = TileRows * Rank / 16 / 64 / Movers;
    static constexpr int TailLoads = Movers <= Parts ? Parts / Movers : 1;
    struct Codes {
        u32x4 w[MainLoads + TailLoads];
        uint32_t scale[MainLoads + TailLoads];
    };
    // Part, row in it and 16 codes of load i; false: none for this lane.
    __device__ __forceinline__ bool unit(int i, int mover, int &part, int &r, int &u) const
    {
        if (i < MainLoads) {
            constexpr int Units = Rank / 16, PerLoad = 64 / Units;   // of a row; rows of a load
            const int row = (i * Movers + mover) * PerLoad + lane / Units;
            part = (i * Movers + mover) * PerLoad / 16, r = row & 15, u = lane & (Units - 1);
            return true;
        }
        u = Rank / 16 + (lane & (2 * RO - 1));
        if constexpr (Movers <= Parts) {
            part = (i - MainLoads) * Movers + mover, r = lane / (2 * RO) & 15;
            return lane < 32 * RO;
        } else {   // eight rows a wave
            part = mover >> 1, r = 8 * (mover & 1) + (lane / (2 * RO) & 7);
            return lane < 16 * RO;
        }
    }
    __device__ __forceinline__ void fetch_codes(const Where &w, int mover, Codes &c) const
    {
        const uint32_t stride = (uint32_t)la.c.token_stride, sstride = (uint32_t)la.c.stoken_stride;
#pragma unroll
        for (int i = 0; i < MainLoads + TailLoads; ++i) {
            int part, r, u;
            if (!unit(i, mover, part, r, u)) continue;
            const bool main = i < MainLoads;
            // the load's rows of all waves begin in part `at`, and may end in the next one
            constexpr int Rows = Movers * (64 / (Rank / 16));
            const int at = main ? i * Rows / 16 : (i - MainLoads) * Movers;
            const bool next = main && Rows > 16 && part != at;
            const int64_t from = main || Movers == 1 ? (next ? w.at[(at + 1) % Parts] : w.at[at]) : w.mine;
            const int64_t sfrom = main || Movers == 1 ? (next ? w.sat[(at + 1) % Parts] : w.sat[at]) : w.smine;
            const uint32_t row = row_of(w.last, part, r);
            c.w[i] = *reinterpret_cast<const u32x4 *>(la.c.rows + from + (row * stride + u * 16));
            c.scale[i] = (la.c.scale + sfrom)[row * sstride + (u >> 1)];
        }
    }
    __device__ __forceinline__ void put_codes(const Codes &c, int mover, char *tile) const
    {
#pragma unroll
        for (int i = 0; i < MainLoads + TailLoads; ++i) {
            int part, r, u;
            if (!unit(i, mover, part, r, u)) continue;
            const float s = scale_of(c.scale[i]);
            const int row = 16 * part + r;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = c.w[i][2 * h], w1 = c.w[i][2 * h + 1];
                const u32x4 y = {codes_to_bf16x2<KVR_KV_FP8, 0>(w0, s), codes_to_bf16x2<KVR_KV_FP8, 1>(w0, s),
                                 codes_to_bf16x2<KVR_KV_FP8, 0>(w1, s), codes_to_bf16x2<KVR_KV_FP8, 1>(w1, s)};
                const int ch = 2 * u + h;
                char *to = i < MainLoads ? tile + row * (Rank * 2) + ((ch ^ r) << 4)
                                         : tile + Main + row * (64 * RO) + (((ch - Rank / 8) ^ tail_swizzle(r)) << 4);
                *reinterpret_cast<u32x4 *>(to) = y;
            }
        }
    }

    // ---- fragments from LDS --------------------------------------------------------------------

    // Block i of 16 rows from row 16 t on, along the rows: chunk 4 i + g, of whose number the lower
    // bits change places with the row's.
    template <int I, int T>
    __device__ __forceinline__ static u32x4 key_fragment(const char *tile, uint32_t key_at, uint32_t tail_at)
    {
        if constexpr (I < RK)
            return *reinterpret_cast<const u32x4 *>(tile + (key_at ^ (I & 3) << 6) + (I >> 2) * 256 + T * 16 * Rank * 2);
        else
            return *reinterpret_cast<const u32x4 *>(tile + (tail_at ^ (I - RK) << 6) + T * 16 * 64 * RO);
    }
    // Columns 16 e on of 32 rows from `tile` on, across the rows; e = 8 E8 + E1.
    template <int E1>
    __device__ __forceinline__ static u32x4 val_fragment(const char *tile, uint32_t val_at)
    {
        const char *p = tile + (val_at ^ E1 << 5);
        const u32x2 lo = read_across(p), hi = read_across(p + 16 * Rank * 2);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }

    // Infinities and NaN in columns c0 chunks on, `Chunks` of them, of a tile's latents: whether there
    // are any (a weight of zero would not hide them), and to zero once the scores have been formed;
    // put_odd() puts them back for the rows that see them.  (A row's chunks change places among 16.)
    template <int Chunks>
    __device__ __forceinline__ bool has_odd(const char *tile, int c0) const
    {
        u16x2 most = {0, 0};
#pragma unroll 4
        for (int i = lane; i < TileRows * Chunks; i += 64) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(tile + i / Chunks * (Rank * 2) + (c0 + (i & (Chunks - 1))) * 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) keep_most<MT>(x[k], most);
        }
        return any_odd<MT>(most);
    }
    template <int Chunks>
    __device__ __forceinline__ void clear_odd(char *tile, int c0) const
    {
#pragma unroll 1
        for (int i = lane; i < TileRows * Chunks; i += 64) {
            u32x4 *at = reinterpret_cast<u32x4 *>(tile + i / Chunks * (Rank * 2) + (c0 + (i & (Chunks - 1))) * 16);
            const u32x4 x = *at;
            uint32_t w[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int k = 0; k < 4; ++k) clear_odd2<MT>(w[k]);
            *at = u32x4{w[0], w[1], w[2], w[3]};
        }
    }

    // ---- which rows see what ---------------------------------------------------------------------

    __device__ __forceinline__ bool sees(int i, int j) const   // query i, newest token j
    {
        if (j < 0) return true;
        if (a.mask) return (a.mask[(int64_t)(q0 + i) * a.words + (j >> 6)] >> (j & 63)) & 1;
        return j <= i;
    }
    // Which of tokens t to t + 3 before `end` query i sees, as bits; word: its mask, if that is one word.
    __device__ __forceinline__ uint32_t seen4(int i, uint64_t word, int t, int end) const
    {
        const int j = t - prefix;
        uint32_t s;
        if (!a.mask) {
            s = (16u >> (3 - max(-1, min(i - j, 3)))) - 1;   // the lowest i - j + 1 bits
        } else if (a.words == 1) {
            const int up = max(0, min(-j, 4));   // older tokens among the four
            s = (uint32_t)(word >> max(0, min(j, 63))) << up | ((1u << up) - 1);
            if (j > 63) s = 0;
        } else {
            s = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) s |= (t + k < end && sees(i, j + k) ? 1u : 0u) << k;
        }
        return s & ((1u << max(0, min(end - t, 4))) - 1);
    }
    // The scores of tokens that are hidden from query i to -infinity; t: the lane's first token.
    __device__ __forceinline__ void hide(int i, int t, int end, f32x4 (&sc)[2]) const
    {
        const uint64_t word = a.mask && a.words == 1 ? a.mask[q0 + i] : 0;
        const uint32_t seen = seen4(i, word, t, end) | seen4(i, word, t + 16, end) << 4;
        const f32x4 x = sc[0], y = sc[1];
        auto pick = [&](int k, float z) { return seen >> k & 1 ? z : -INFINITY; };
        sc[0] = f32x4{pick(0, x[0]), pick(1, x[1]), pick(2, x[2]), pick(3, x[3])};
        sc[1] = f32x4{pick(4, y[0]), pick(5, y[1]), pick(6, y[2]), pick(7, y[3])};
    }

    // References move only when a score exceeds the last maximum that they were taken from by
    // more than 8 (weights of up to 2^8 lose no precision); in half precision they stand 2^7 below
    // it, so that weights that vanish are below 2^-32 of the row's largest.
    static constexpr float kBelow = MT == KVR_DT_FP16 ? 7.0f : 0.0f;

    __device__ __forceinline__ float largest(const f32x4 (&sc)[2]) const
    {
        const f32x4 x = sc[0], y = sc[1];
        return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))) *
               a.scale2;
    }
    // Eight weights against reference m, rounded to the products' type; sums of them as they are
    // and as rounded (what the outputs are divided by).
    __device__ __forceinline__ u32x4 weights(const f32x4 (&sc)[2], float m, float &sum, float &rounded) const
    {
        const f32x4 s0 = sc[0], s1 = sc[1];
        float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -m));
        sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        uint32_t w[4];
        rounded = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack16<MT>(x[2 * i], x[2 * i + 1]);
            rounded = add_pair<MT>(w[i], rounded);
        }
        return u32x4{w[0], w[1], w[2], w[3]};
    }

    // The query of row `row` of the sequence, rows past the last as that one; its fragments.
    __device__ __forceinline__ int query_of(int row) const { return min(row, rows - 1) / a.group; }
    __device__ __forceinline__ void load_query(int row, u32x4 (&q)[NB]) const
    {
        const int i0 = query_of(row), head = min(row, rows - 1) - i0 * a.group;
        const char *src = a.q.p + ((int64_t)(q0 + i0) * a.q.token_stride + (int64_t)head * a.q.head_stride) * 2;
        static_for<0, NB>([&](auto I) {
            constexpr int i = decltype(I)::value;
            q[i] = *reinterpret_cast<const u32x4 *>(src + (i * 32 + g * 8) * 2);
        });
        __builtin_amdgcn_sched_barrier(0);   // all loads first
    }
    __device__ __forceinline__ static void negate(u32x4 (&q)[NB])
    {
        static_for<0, NB>([&](auto I) { q[decltype(I)::value] ^= 0x80008000u; });
    }

    // ---- results --------------------------------------------------------------------------------

    // Four elements from d on of row r0 + row of the output, divided by norm, or of a part's.
    __device__ __forceinline__ void store(const Part &p, int r0, int row, int block_rows, int d, f32x4 x,
                                          float inv) const
    {
        if (p.parts != 1) {
            *reinterpret_cast<f32x4 *>(a.part_o + ((int64_t)item * block_rows + row) * Rank + d) = x;
            return;
        }
        const int i0 = (r0 + row) / a.group, head = r0 + row - i0 * a.group;
        char *y = a.out.p + ((int64_t)(q0 + i0) * a.out.token_stride + (int64_t)head * a.out.head_stride + d) * 2;
        *reinterpret_cast<u32x2 *>(y) = u32x2{pack16<MT>(x[0] * inv, x[1] * inv), pack16<MT>(x[2] * inv, x[3] * inv)};
    }
    __device__ __forceinline__ void store_sums(const Part &p, int r0, int row, int block_rows, float top,
                                               float sum, float norm) const
    {
        if (p.parts != 1) {
            a.part_ml[(int64_t)item * block_rows + row] = float4{top, sum, norm, 0.0f};
        } else if (a.lse) {
            const int i0 = (r0 + row) / a.group, head = r0 + row - i0 * a.group;
            a.lse[(int64_t)(q0 + i0) * a.q_heads + head] =
                sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }

    // Whether element d of token t's latent is an infinity or a NaN.
    __device__ __forceinline__ bool odd_at(int t, int d) const
    {
        int id = pages[t >> a.c.page_shift];
        if (id < 0 || id >= a.c.n_pages) id = 0;
        const int off = t & ((1 << a.c.page_shift) - 1);
        const char *row = la.c.rows + id * la.c.page_stride + off * la.c.token_stride;
        uint32_t bits;
        if (Quant) {
            const uint32_t sc = la.c.scale[id * la.c.spage_stride + off * la.c.stoken_stride + (d >> 5)];
            bits = codes_to_bf16x2<KVR_KV_FP8, 0>(reinterpret_cast<const uint8_t *>(row)[d], scale_of(sc)) & 0xffffu;
        } else {
            bits = reinterpret_cast<const uint16_t *>(row)[d];
        }
        constexpr uint32_t e = MT == KVR_DT_FP16 ? 0x7c00u : 0x7f80u;
        return (bits & e) == e;
    }
    // What was taken out of the products where tokens are hidden, to the block's rows that see it,
    // after they have been stored.  The same element was part of the score: that is an infinity or a
    // NaN too, the weight 0 or NaN, and their product NaN.  A tile is cleared whole if it holds a token
    // that some query may not see, or ends past the part: all of the part's tokens are looked at from
    // the first such tile on, older ones among them.
    __device__ __forceinline__ void put_odd(const Part &p, int r0, int block_rows) const
    {
        wait_loads<0>();   // of stores too
        __syncthreads();
        const int t0 = p.first * kStep, t1 = min(len, p.last * kStep);
        const int from = t0 + max(0, min(prefix, t1) - t0) / TileRows * TileRows;
        for (int i = threadIdx.x; i < min(block_rows, rows - r0) * Rank; i += blockDim.x) {
            const int row = i / Rank, d = i - row * Rank;
            const int i0 = (r0 + row) / a.group;
            for (int t = from; t < t1; ++t) {
                if (!sees(i0, t - prefix) || !odd_at(t, d)) continue;
                if (p.parts != 1) {
                    a.part_o[((int64_t)item * block_rows + row) * Rank + d] = __uint_as_float(0x7fc00000u);
                } else {
                    const int head = r0 + row - i0 * a.group;
                    uint16_t *y = reinterpret_cast<uint16_t *>(a.out.p) +
                                  (int64_t)(q0 + i0) * a.out.token_stride + (int64_t)head * a.out.head_stride;
                    y[d] = 0x7fff;
                }
                break;
            }
        }
    }
};

// Runs Keys fragments through `key`, then middle(), then Vals through `val`; load(k) reads fragment
// k, G at a time and a group ahead of their use.  (middle() says whether it has changed the tile.)
template <int G, int Keys, int Vals, class Load, class Key, class Middle, class Val>
__device__ __forceinline__ void fragments(Load load, Key key, Middle middle, Val val)
{
    constexpr int KG = (Keys + G - 1) / G, VG = (Vals + G - 1) / G;
    u32x4 frag[2][G];
    auto fetch = [&](auto K) {
        constexpr int k = decltype(K)::value;
        static_for<0, G>([&](auto J) {
            constexpr int j = decltype(J)::value;
            constexpr int at = k < KG ? k * G + j : Keys + (k - KG) * G + j;
            if constexpr (k < KG ? at < Keys : at < Keys + Vals)
                frag[k & 1][j] = load(std::integral_constant<int, at>{});
        });
        __builtin_amdgcn_sched_barrier(0x406);   // only vector and scalar arithmetic may pass
    };
    fetch(std::integral_constant<int, 0>{});
    static_for<0, KG>([&](auto K) {
        constexpr int k = decltype(K)::value;
        if constexpr (k + 1 < KG + VG) fetch(std::integral_constant<int, k + 1>{});
        static_for<0, G>([&](auto J) {
            constexpr int j = decltype(J)::value, at = k * G + j;
            if constexpr (at < Keys) key(std::integral_constant<int, at>{}, frag[k & 1][j]);
        });
    });
    if (middle()) fetch(std::integral_constant<int, KG>{});
    static_for<0, VG>([&](auto K) {
        constexpr int k = KG + decltype(K)::value;
        if constexpr (k + 1 < KG + VG) fetch(std::integral_constant<int, k + 1>{});
        static_for<0, G>([&](auto J) {
            constexpr int j = decltype(J)::value, at = decltype(K)::value * G + j;
            if constexpr (at < Vals) val(std::integral_constant<int, at>{}, frag[k & 1][j]);
        });
    });
}

// ---- up to 16 rows ----------------------------------------------------------------------------

template <int FMT, int RK, int RO>
struct FewRows : LatentTile<FMT, RK, RO, 32, 1> {
    using T = LatentTile<FMT, RK, RO, 32, 1>;
    using T::a, T::n, T::g, T::lane, T::len, T::prefix, T::rows;
    static constexpr int MT = T::MT, Rank = T::Rank, NB = T::NB, Waves = 4, BlockRows = 16;
    static constexpr int JoinRow = Rank + 4;   // floats
    static constexpr int JoinBytes = Waves * 16 * JoinRow * 4, TileBytes = Waves * T::Tile;
    static constexpr int StatsAt = TileBytes > JoinBytes ? TileBytes : JoinBytes;
    static constexpr int LdsBytes = StatsAt + 3 * (Waves + 1) * 16 * 4 + 16;

    u32x4 q[NB];
    f32x4 o[2 * RK];
    float m, l, w;   // reference (log2); this lane's part of the sum of the weights, and as rounded

    __device__ FewRows(const LatentAttention &la) : T(la) {}

    __device__ __forceinline__ bool compute(int step, int query, char *tile)
    {
        // (Opaque, or the compiler forms every chunk's address before the loop, in registers that
        // it does not have.)
        uint32_t key_at = T::key_at, tail_at = T::tail_at, val_at = T::val_at;
        asm volatile("" : "+v"(key_at), "+v"(tail_at), "+v"(val_at));
        const bool hides = (step + 1) * kStep > prefix;
        const bool odd = hides && T::template has_odd<Rank / 8>(tile, 0);
        f32x4 sc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
        u32x4 pv;
        auto load = [&](auto K) {
            constexpr int k = decltype(K)::value, e = k - 2 * NB;
            if constexpr (k < 2 * NB) return T::template key_fragment<k / 2, k % 2>(tile, key_at, tail_at);
            else return T::template val_fragment<(e & 7)>(tile + (e >> 3) * 256, val_at);
        };
        auto key = [&](auto K, u32x4 x) {
            constexpr int k = decltype(K)::value;
            sc[k % 2] = mfma<MT>(x, q[k / 2], sc[k % 2]);
        };
        auto middle = [&] {
            if (hides) T::hide(query, step * kStep + 4 * g, len, sc);
            const float top = T::largest(sc);
            if (__ballot(top > m + (8.0f + T::kBelow))) {
                const float t = fmaxf(row_max(top) - T::kBelow, m);
                const float f = __builtin_amdgcn_exp2f(m - t);
                l *= f;
                w *= f;
                static_for<0, 2 * RK>([&](auto E) { o[decltype(E)::value] *= f; });
                m = t;
            }
            float sum, rounded;
            pv = T::weights(sc, m, sum, rounded);
            l += sum;
            w += rounded;
            if (odd) T::template clear_odd<Rank / 8>(tile, 0);
            return odd;
        };
        auto val = [&](auto E, u32x4 x) {
            constexpr int e = decltype(E)::value;
            o[e] = mfma<MT>(x, pv, o[e]);
        };
        fragments<8, 2 * NB, 2 * RK>(load, key, middle, val);
        return odd;
    }

    __device__ __forceinline__ void run(char *lds)
    {
        const Part p = T::find();
        if (p.b < 0) return;
        T::begin(p);
        const int wave = uniform((int)(threadIdx.x >> 6));
        const int r0 = p.rb * BlockRows, query = T::query_of(r0 + n);
        char *tile = lds + wave * T::Tile;
        const uint32_t tile_at = lds_address(tile);
        int s = p.first + wave;
        T::load_query(r0 + n, q);
        T::hold(p.first * kStep >> a.c.page_shift);
        typename T::Codes c;
        if (s < p.last) {
            if constexpr (T::Quant) T::fetch_codes(T::locate(s * kStep, len, 0), 0, c);
            else T::fetch(T::locate(s * kStep, len, 0), 0, tile_at);
        }
        if (a.negate) T::negate(q);
        m = kLowest, l = 0.0f, w = 0.0f;
        static_for<0, 2 * RK>([&](auto E) { o[decltype(E)::value] = f32x4{0, 0, 0, 0}; });
        bool odd = false;
        for (; s < p.last; s += Waves) {
            if constexpr (T::Quant) {
                T::put_codes(c, 0, tile);
                if (s + Waves < p.last) T::fetch_codes(T::locate((s + Waves) * kStep, len, 0), 0, c);
            } else {
                wait_loads<0>();
            }
            odd |= compute(s, query, tile);
            if constexpr (!T::Quant) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
                if (s + Waves < p.last) T::fetch(T::locate((s + Waves) * kStep, len, 0), 0, tile_at);
            }
        }
        // Join the waves: maxima first; then values, and by one wave the sums, in their order.
        float *sm = reinterpret_cast<float *>(lds + StatsAt), *sl = sm + Waves * 16, *sw = sl + Waves * 16;
        float *total = sw + Waves * 16;   // of each row: maximum, sum, sum as rounded
        l = row_sum(l);
        w = row_sum(w);
        if (g == 0) {
            sm[wave * 16 + n] = m;
            sl[wave * 16 + n] = l;
            sw[wave * 16 + n] = w;
        }
        odd = block_any(odd, reinterpret_cast<uint32_t *>(lds + LdsBytes - 16));
        float top = kLowest;
#pragma unroll
        for (int t = 0; t < Waves; ++t) top = fmaxf(top, sm[t * 16 + n]);
        const float f = __builtin_amdgcn_exp2f(m - top);
        float *row = reinterpret_cast<float *>(lds) + (wave * 16 + n) * JoinRow + 4 * g;
        static_for<0, 2 * RK>([&](auto E) {
            *reinterpret_cast<f32x4 *>(row + 16 * decltype(E)::value) = o[decltype(E)::value] * f;
        });
        if (wave == 0 && g == 0) {
            float sum = 0.0f, norm = 0.0f;
#pragma unroll
            for (int t = 0; t < Waves; ++t) {
                const float h = __builtin_amdgcn_exp2f(sm[t * 16 + n] - top);
                sum += sl[t * 16 + n] * h;
                norm += sw[t * 16 + n] * h;
            }
            total[n] = top;
            total[16 + n] = sum;
            total[32 + n] = norm;
        }
        __syncthreads();
        const float *so = reinterpret_cast<const float *>(lds);
        constexpr int PerRow = Rank / 4, Rounds = 16 * PerRow / (64 * Waves);
#pragma unroll
        for (int i = 0; i < Rounds; ++i) {
            const int at = i * 64 * Waves + threadIdx.x, r = at / PerRow, d = 4 * (at & (PerRow - 1));
            if (r0 + r >= rows) continue;
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < Waves; ++t) x += *reinterpret_cast<const f32x4 *>(so + (t * 16 + r) * JoinRow + d);
            const float norm = total[32 + r];
            T::store(p, r0, r, BlockRows, d, x, norm == 0.0f ? 0.0f : 1.0f / norm);
            if (d == 0) T::store_sums(p, r0, r, BlockRows, total[r], total[16 + r], norm);
        }
        if (odd) T::put_odd(p, r0, BlockRows);
    }
};

// ---- more rows ----------------------------------------------------------------------------------

template <int FMT, int RK, int RO, int RT, int WAVES>
struct ManyRows : LatentTile<FMT, RK, RO, 64, WAVES> {
    using T = LatentTile<FMT, RK, RO, 64, WAVES>;
    using T::a, T::n, T::g, T::lane, T::len, T::prefix, T::rows;
    static constexpr int MT = T::MT, NB = T::NB, Waves = WAVES, Groups = Waves / 2, BlockRows = Groups * 16 * RT;
    static constexpr int VT = RK;   // value tiles of a wave: half of the columns
    static constexpr int Group = WAVES == 4 ? 8 : RT == 2 ? 2 : 4;   // fragments, as registers allow
    // LDS: two tiles, the weights that waves exchange, what they say about their references
    static constexpr int WeightsAt = 2 * T::Tile, MaxAt = WeightsAt + Waves * RT * 1024;
    static constexpr int FlagAt = MaxAt + Waves * RT * 16 * 4, LdsBytes = FlagAt + 16;

    u32x4 q[RT][NB];
    f32x4 o[RT][VT];
    float m[RT], l[RT], w[RT];
    int wave, side;   // side: which half of the cached rows, and of the columns

    __device__ ManyRows(const LatentAttention &la) : T(la) {}

    // Row of the block's that lane n has in this wave's tile r: the tiles of a group are as many rows
    // apart as all groups have, so that each has one before any has two.
    __device__ __forceinline__ int row_in_block(int r) const { return 16 * ((wave >> 1) + Groups * r) + n; }

    // Step k of the block: rows t to t + 63, before `end`.  R: this wave's tiles with any rows.
    template <int R>
    __device__ __forceinline__ bool compute(int k, int t, int end, int r0, char *tile, char *lds)
    {
        uint32_t *flag = reinterpret_cast<uint32_t *>(lds + FlagAt) + (k & 1);
        if constexpr (R == 0) {   // the others' barriers
            block_barrier();
            if (*flag == (uint32_t)k + 1) {
                block_barrier();
                block_barrier();
            }
            return false;
        } else {
        uint32_t key_at = T::key_at, tail_at = T::tail_at, val_at = T::val_at;
        asm volatile("" : "+v"(key_at), "+v"(tail_at), "+v"(val_at));
        const bool hides = t + 64 > prefix || t + 64 > end;
        // this wave's rows for the scores, and columns for the outputs
        const char *mine = tile + side * 32 * T::Rank * 2, *mine_tail = tile + side * 32 * 64 * RO;
        const char *half = tile + side * (T::Rank / 16 >> 3) * 128;
        const bool odd = hides && T::template has_odd<T::Rank / 16>(tile, side * (T::Rank / 16));
        f32x4 sc[R][2];
        u32x4 pv[R][2];   // weights of the first and the second 32 rows
        static_for<0, 2 * R>([&](auto I) {
            sc[decltype(I)::value / 2][decltype(I)::value % 2] = f32x4{0, 0, 0, 0};
        });
        u32x4 *shared = reinterpret_cast<u32x4 *>(lds + WeightsAt) + lane;
        auto load = [&](auto K) {
            constexpr int f = decltype(K)::value, e = f - 2 * NB;   // e: tile, then half of the rows
            if constexpr (f < 2 * NB && f / 2 < RK) return T::template key_fragment<f / 2, f % 2>(mine, key_at, tail_at);
            else if constexpr (f < 2 * NB) return T::template key_fragment<f / 2, f % 2>(mine_tail, key_at, tail_at);
            else return T::template val_fragment<(e / 2 & 7)>(half + (e / 2 >> 3) * 256 + (e & 1) * 32 * T::Rank * 2, val_at);
        };
        auto key = [&](auto K, u32x4 x) {
            constexpr int f = decltype(K)::value;
            static_for<0, R>([&](auto I) {
                constexpr int r = decltype(I)::value;
                sc[r][f % 2] = mfma<MT>(x, q[r][f / 2], sc[r][f % 2]);
            });
        };
        auto middle = [&] {
            float top[R], sum[R], rounded[R];
            bool moves = false;
            static_for<0, R>([&](auto I) {
                constexpr int r = decltype(I)::value;
                if (hides) T::hide(T::query_of(r0 + row_in_block(r)), t + 32 * side + 4 * g, end, sc[r]);
                top[r] = T::largest(sc[r]);
                moves = moves || top[r] > m[r] + (8.0f + T::kBelow);
            });
            auto weigh = [&] {
                static_for<0, R>([&](auto I) {
                    constexpr int r = decltype(I)::value;
                    const u32x4 p = T::weights(sc[r], m[r], sum[r], rounded[r]);
                    shared[(wave * RT + r) * 64] = p;
                    pv[r][0] = p;
                });
            };
            weigh();
            if (__ballot(moves) && lane == 0) *flag = (uint32_t)k + 1;
            block_barrier();
            if (*flag == (uint32_t)k + 1) {   // some reference moves: the two waves of a row agree on theirs
                float *rm = reinterpret_cast<float *>(lds + MaxAt);
                static_for<0, R>([&](auto I) {
                    constexpr int r = decltype(I)::value;
                    top[r] = row_max(top[r]);
                    if (g == 0) rm[(wave * RT + r) * 16 + n] = top[r];
                });
                block_barrier();
                static_for<0, R>([&](auto I) {
                    constexpr int r = decltype(I)::value;
                    const float x = fmaxf(fmaxf(top[r], rm[((wave ^ 1) * RT + r) * 16 + n]) - T::kBelow, m[r]);
                    const float f = __builtin_amdgcn_exp2f(m[r] - x);
                    l[r] *= f;
                    w[r] *= f;
                    static_for<0, VT>([&](auto E) { o[r][decltype(E)::value] *= f; });
                    m[r] = x;
                });
                weigh();
                block_barrier();
            }
            static_for<0, R>([&](auto I) {
                constexpr int r = decltype(I)::value;
                l[r] += sum[r];
                w[r] += rounded[r];
                const u32x4 other = shared[((wave ^ 1) * RT + r) * 64], own = pv[r][0];
                pv[r][0] = side ? other : own;
                pv[r][1] = side ? own : other;
            });
            // (all scores have been formed; the other wave with these columns writes the same)
            if (odd) T::template clear_odd<T::Rank / 16>(tile, side * (T::Rank / 16));
            return odd;
        };
        auto val = [&](auto E, u32x4 x) {
            constexpr int e = decltype(E)::value;
            static_for<0, R>([&](auto I) {
                constexpr int r = decltype(I)::value;
                o[r][e / 2] = mfma<MT>(x, pv[r][e & 1], o[r][e / 2]);
            });
        };
        fragments<Group, 2 * NB, 2 * VT>(load, key, middle, val);
        return odd;
        }
    }

    __device__ __forceinline__ void run(char *lds)
    {
        const Part p = T::find();
        if (p.b < 0) return;
        T::begin(p);
        wave = uniform((int)(threadIdx.x >> 6)), side = wave & 1;
        const int r0 = p.rb * a.block_rows, mine = min(a.block_rows, rows - r0);   // the block's rows
        const int tiles = min(RT, (mine - 16 * (wave >> 1) + 16 * Groups - 1) / (16 * Groups));   // of this wave
        const int first = p.first * kStep, end = min(len, p.last * kStep);
        const int steps = (end - first + 63) / 64;
        const uint32_t lds_at = lds_address(lds);
        static_for<0, RT>([&](auto R) { T::load_query(r0 + row_in_block(decltype(R)::value), q[decltype(R)::value]); });
        T::hold(p.first * kStep >> a.c.page_shift);
        typename T::Codes c;
        if constexpr (T::Quant) T::fetch_codes(T::locate(first, end, wave), wave, c);
        else T::fetch(T::locate(first, end, wave), wave, lds_at);
        if (threadIdx.x < 2) reinterpret_cast<uint32_t *>(lds + FlagAt)[threadIdx.x] = 0;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            if (a.negate) T::negate(q[r]);
            m[r] = kLowest, l[r] = 0.0f, w[r] = 0.0f;
            static_for<0, VT>([&](auto E) { o[r][decltype(E)::value] = f32x4{0, 0, 0, 0}; });
        });
        bool odd = false;
        auto loop = [&](auto R) {
            for (int k = 0; k < steps; ++k) {
                const int t = first + 64 * k;
                char *tile = lds + (k & 1) * T::Tile;
                if constexpr (T::Quant) {
                    T::put_codes(c, wave, tile);
                    if (k + 1 < steps) T::fetch_codes(T::locate(t + 64, end, wave), wave, c);
                } else {
                    wait_loads<0>();
                }
                block_barrier();   // the step's rows are there, the other tile has been read
                if constexpr (!T::Quant)
                    if (k + 1 < steps) T::fetch(T::locate(t + 64, end, wave), wave, lds_at + ((k + 1) & 1) * T::Tile);
                odd |= compute<decltype(R)::value>(k, t, end, r0, tile, lds);
            }
        };
        // (loops of their own, or the registers of all are live in each; the barriers are the same)
        if (RT == 2 && tiles == 2) loop(std::integral_constant<int, RT>{});
        else if (tiles > 0) loop(std::integral_constant<int, 1>{});
        else loop(std::integral_constant<int, 0>{});
        __syncthreads();   // LDS may be used for other things
        odd = block_any(odd, reinterpret_cast<uint32_t *>(lds + FlagAt));
        // the sums of a row's two waves
        float *sums = reinterpret_cast<float *>(lds);
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            l[r] = row_sum(l[r]);
            w[r] = row_sum(w[r]);
            if (g == 0) {
                sums[(2 * wave * RT + r) * 16 + n] = l[r];
                sums[((2 * wave + 1) * RT + r) * 16 + n] = w[r];
            }
        });
        __syncthreads();
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const int row = row_in_block(r);
            if (row >= mine) return;
            const float sum = l[r] + sums[(2 * (wave ^ 1) * RT + r) * 16 + n];
            const float norm = w[r] + sums[((2 * (wave ^ 1) + 1) * RT + r) * 16 + n];
            const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
            static_for<0, VT>([&](auto E) {
                constexpr int e = decltype(E)::value;
                T::store(p, r0, row, a.block_rows, side * (T::Rank / 2) + 16 * e + 4 * g, o[r][e], inv);
            });
            if (side == 0 && g == 0) T::store_sums(p, r0, row, a.block_rows, m[r], sum, norm);
        });
        if (odd) T::put_odd(p, r0, a.block_rows);
    }
};

// With eight waves a block two share a SIMD's registers.
template <class K>
__global__ __launch_bounds__(64 * K::Waves, K::Waves / 4) void latent_kernel(LatentAttention l)
{
    __shared__ __align__(1024) char lds[K::LdsBytes];
    K k(l);
    k.run(lds);
}

template <class K>
hipError_t launch_latent_kernel(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    if (l.a.block_rows > K::BlockRows) return hipErrorInvalidValue;
    latent_kernel<K><<<grid, 64 * K::Waves, 0, stream>>>(l);
    return hipGetLastError();
}

template <int FMT, int RK, int RO>
hipError_t launch_latent_rows(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    const int n = l.a.block_rows;   // as plan_latent_attention chose
    if (n <= 16) return launch_latent_kernel<FewRows<FMT, RK, RO>>(l, grid, stream);
    if (n <= 32) return launch_latent_kernel<ManyRows<FMT, RK, RO, 1, 4>>(l, grid, stream);
    if (n <= 64) return launch_latent_kernel<ManyRows<FMT, RK, RO, 1, 8>>(l, grid, stream);
    if constexpr (RK == 8) return launch_latent_kernel<ManyRows<FMT, RK, RO, 2, 8>>(l, grid, stream);
    else return hipErrorInvalidValue;
}

template <int FMT>
hipError_t launch_latent_format(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    const bool wide = l.c.rot == 64;
    if (l.c.rank == 512)
        return wide ? launch_latent_rows<FMT, 16, 2>(l, grid, stream) : launch_latent_rows<FMT, 16, 1>(l, grid, stream);
    return wide ? launch_latent_rows<FMT, 8, 2>(l, grid, stream) : launch_latent_rows<FMT, 8, 1>(l, grid, stream);
}

}  // namespace
}  // namespace kv
}  // namespace kvr
