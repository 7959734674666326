// Attention over the latent cache (the absorbed form):
//   out_r = sum_j p_rj x_j[: rank] / sum_j p_rj,   p_rj = exp(scale q_r . x_j - m_r),
// one pass over the cached rows x_j with the running maximum m_r and sum.  A row r is one head
// of one new token; all of them share the cached rows.
//
// Matrix instructions (16x16x32) compute S^T = X Q^T and O^T = X[: rank]^T P^T, so that a lane
// owns one row r (lane mod 16) throughout and P^T leaves the first product in the layout that
// the second one takes.  32 cached rows (a step) lie in LDS as they lie in memory, 16-byte
// chunks exchanged within a row so that neither reading disturbs the banks; the first
// product reads them along the row, the second one across (ds_read_b64_tr_b16 turns 4x16
// elements around).  So a cached row is fetched once and is key and value.  16-bit rows go from
// memory to LDS without passing through registers; codes are converted to bfloat16 on the way,
// exactly.
//
// A block has four waves.  WR of them share the rows of the cache and divide the queries, 16
// RT rows each; 4 / WR such groups take every n-th step.  Up to 32 rows each wave is a group of
// its own, which needs no barrier and leaves the three others' loads in flight while it computes
// (memory bounds this); beyond, waves share what is fetched, because LDS can be read
// about as fast as 32 rows a wave can use it.
//
// Each source that includes this header builds the kernel for one cache format.
#pragma once

#include "kvr_attention.h"
#include "kvr_latent.h"

namespace kvr {
namespace kv {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) uint32_t lds_u32;
typedef __attribute__((address_space(1))) const uint32_t global_u32;

// 16 bytes a lane from p into LDS: lane l's at `to` (uniform) + 16 l.
__device__ __forceinline__ void load_to_lds(const char *p, char *to)
{
    __builtin_amdgcn_global_load_lds((global_u32 *)p, (lds_u32 *)to, 16, 0, 0);
}
// Waits for all of this wave's loads.
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("" ::: "memory");
}

// Four elements of this lane's column (lane mod 16) of a block of four rows and 16 columns; p:
// columns 4 (lane mod 4) on of row lane / 4 mod 4.
__device__ __forceinline__ u32x2 read_across(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// Infinities and NaN of two 16-bit values to zero; whether there was one.
template <int MT>
__device__ __forceinline__ bool clear_odd2(uint32_t &x)
{
    constexpr uint32_t e = MT == KVR_DT_FP16 ? 0x7c00u : 0x7f80u;
    bool odd = false;
    if ((x & e) == e) x &= 0xffff0000u, odd = true;
    if ((x & e << 16) == e << 16) x &= 0xffffu, odd = true;
    return odd;
}

template <int FMT, int RK, int RO, int RT, int WR>
struct LatentKernel {
    static constexpr int Rank = 32 * RK, NB = RK + RO;      // blocks of 32 elements of a row
    static constexpr bool Quant = FMT == KVR_KV_FP8;
    static constexpr int MT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // product type
    static constexpr int Waves = 4, WT = Waves / WR;        // WT: groups of waves
    static constexpr int GroupRows = 16 * RT * WR, BlockRows = GroupRows;
    static constexpr int Buffers = WR > 1 && !Quant ? 2 : 1;
    // LDS bytes: the latents of a step, its shared keys
    static constexpr int Main = 32 * Rank * 2, Tail = 32 * 32 * RO * 2, Tile = Main + Tail;
    static constexpr int JoinRow = Rank + 4;                // floats
    static constexpr int JoinBytes = WT > 1 ? Waves * 16 * JoinRow * 4 : 0;
    static constexpr int TileBytes = WT * Buffers * Tile;
    static constexpr int StatBytes = 3 * Waves * 16 * RT * 4;
    static constexpr int LdsBytes = (TileBytes > JoinBytes ? TileBytes : JoinBytes) + StatBytes;

    struct State {   // of this wave's rows
        u32x4 q[RT][NB];
        f32x4 o[RT][2 * RK];
        float m[RT], l[RT];   // reference (log2), this lane's part of the weights' sum
        f32x4 w[RT];          // sum of the rounded weights (every element the same)
        int qi[RT];           // query within the sequence
        uint64_t word[RT];    // its tree mask, where that is one word
    };

    const LatentAttention &la;
    const Attention &a;
    const int n, g, lane;
    int len, prefix, q0;
    const int32_t *pages;
    uint32_t key_at[4], tail_at[RO], val_at[8];   // byte offsets of this lane in a tile

    __device__ LatentKernel(const LatentAttention &l)
        : la(l), a(l.a), n(threadIdx.x & 15), g((threadIdx.x & 63) >> 4), lane(threadIdx.x & 63)
    {
        // Chunk c of row r lies at c ^ (r mod 16) of its row (the latents), c ^ (r / 2 mod 8) or
        // c ^ (r / 4 mod 4) (the shared keys, 8 or 4 chunks): 16 rows' chunks of one column
        // then lie in 16 different places of 256 bytes.
#pragma unroll
        for (int i = 0; i < 4; ++i) key_at[i] = n * (Rank * 2) + (((4 * i + g) ^ n) << 4);
#pragma unroll
        for (int i = 0; i < RO; ++i)
            tail_at[i] = Main + n * (64 * RO) + (((4 * i + g) ^ (RO == 2 ? n >> 1 & 7 : n >> 2 & 3)) << 4);
        const int r = 4 * g + (n >> 2);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            val_at[e] = r * (Rank * 2) + (((2 * e + ((n & 3) >> 1)) ^ r) << 4) + ((n & 1) << 3);
    }

    // ---- a step's rows into LDS ------------------------------------------------------

    // The byte offset of row r of a step in the cache; rows past the end read as the last one.
    struct Where {
        int64_t at[2], sat[2];   // of the first and the second 16 rows
        int last;                // the step's last row
    };
    __device__ __forceinline__ int page_of(int t) const
    {
        int page = __builtin_amdgcn_readfirstlane(pages[t >> a.c.page_shift]);
        if (page < 0 || page >= a.c.n_pages) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            page = 0;
        }
        return page;
    }
    __device__ __forceinline__ Where locate(int step) const
    {
        Where w;
        const int t = step * kStep;
        w.last = min(len - 1 - t, 31);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = i && w.last >= 16 ? t + 16 : t;
            const int page = page_of(u), off = u & ((1 << a.c.page_shift) - 1);
            w.at[i] = page * la.c.page_stride + off * la.c.token_stride;
            w.sat[i] = Quant ? page * la.c.spage_stride + off * la.c.stoken_stride : 0;
        }
        return w;
    }
    __device__ __forceinline__ int64_t row_at(const Where &w, int r) const
    {
        r = min(r, w.last);
        return (r < 16 ? w.at[0] : w.at[1]) + (r & 15) * la.c.token_stride;
    }
    __device__ __forceinline__ int64_t scale_at(const Where &w, int r) const
    {
        r = min(r, w.last);
        return (r < 16 ? w.sat[0] : w.sat[1]) + (r & 15) * la.c.stoken_stride;
    }

    // 16-bit rows: wave `part` of the WR that share a tile brings every WR-th KB.
    __device__ __forceinline__ void fetch(const Where &w, int part, char *tile) const
    {
        constexpr int RowChunks = Rank / 8, TailChunks = 4 * RO;
#pragma unroll
        for (int j0 = 0; j0 < Main / 1024; j0 += WR) {
            const int j = j0 + part;
            const int r = RowChunks == 64 ? j : 2 * j + (lane >> 5);
            const int c = (lane & (RowChunks - 1)) ^ (r & 15);
            load_to_lds(la.c.rows + row_at(w, r) + c * 16, tile + j * 1024);
        }
#pragma unroll
        for (int j0 = 0; j0 < Tail / 1024; j0 += WR) {
            const int j = j0 + part;
            if (Tail / 1024 < WR && j >= Tail / 1024) break;
            const int r = (64 * j + lane) / TailChunks;
            const int c = (lane & (TailChunks - 1)) ^ (RO == 2 ? r >> 1 & 7 : r >> 2 & 3);
            load_to_lds(la.c.rows + row_at(w, r) + Rank * 2 + c * 16, tile + Main + j * 1024);
        }
    }

    // Rows of codes: 16 codes a lane, converted into two chunks.
    static constexpr int CodeUnits = 32 * (Rank + 32 * RO) / 16;
    static constexpr int MainLoads = 32 * Rank / 16 / 64 / WR;              // of a lane
    static constexpr int TailLoads = (32 * 2 * RO + 64 * WR - 1) / (64 * WR);
    struct Codes16 {
        u32x4 w;
        uint32_t scale;
    };
    struct Codes {
        Codes16 x[MainLoads + TailLoads];
    };
    __device__ __forceinline__ void unit(int i, int part, int &r, int &u) const   // unit i of this lane
    {
        if (i < MainLoads) {
            const int at = 64 * (i * WR + part) + lane;
            r = at / (Rank / 16), u = at & (Rank / 16 - 1);
        } else {
            const int at = 64 * ((i - MainLoads) * WR + part) + lane;
            r = at / (2 * RO), u = Rank / 16 + (at & (2 * RO - 1));   // r beyond 31: none
        }
    }
    __device__ __forceinline__ void fetch_codes(const Where &w, int part, Codes &c) const
    {
#pragma unroll
        for (int i = 0; i < MainLoads + TailLoads; ++i) {
            int r, u;
            unit(i, part, r, u);
            if (i >= MainLoads && r > 31) continue;
            c.x[i].w = *reinterpret_cast<const u32x4 *>(la.c.rows + row_at(w, r) + u * 16);
            c.x[i].scale = la.c.scale[scale_at(w, r) + (u >> 1)];
        }
    }
    __device__ __forceinline__ void put_codes(const Codes &c, int part, char *tile) const
    {
#pragma unroll
        for (int i = 0; i < MainLoads + TailLoads; ++i) {
            int r, u;
            unit(i, part, r, u);
            if (i >= MainLoads && r > 31) continue;
            const float s = scale_of(c.x[i].scale);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = c.x[i].w[2 * h], w1 = c.x[i].w[2 * h + 1];
                const u32x4 y = {codes_to_bf16x2<KVR_KV_FP8, 0>(w0, s), codes_to_bf16x2<KVR_KV_FP8, 1>(w0, s),
                                 codes_to_bf16x2<KVR_KV_FP8, 0>(w1, s), codes_to_bf16x2<KVR_KV_FP8, 1>(w1, s)};
                const int ch = 2 * u + h;
                char *to = i < MainLoads
                               ? tile + r * (Rank * 2) + ((ch ^ (r & 15)) << 4)
                               : tile + Main + r * (64 * RO) +
                                     (((ch - Rank / 8) ^ (RO == 2 ? r >> 1 & 7 : r >> 2 & 3)) << 4);
                *reinterpret_cast<u32x4 *>(to) = y;
            }
        }
    }

    // ---- one step ----------------------------------------------------------------------

    __device__ __forceinline__ int token(int step, int i) const   // i of this lane's eight
    {
        return step * kStep + 16 * (i >> 2) + 4 * g + (i & 3);
    }
    __device__ __forceinline__ bool sees(int i, int j) const   // query i, newest token j
    {
        if (j < 0) return true;
        if (a.mask) return (a.mask[(int64_t)(q0 + i) * a.words + (j >> 6)] >> (j & 63)) & 1;
        return j <= i;
    }
    // Which of tokens t to t + 3 the lane's row of tile R sees, as bits.
    template <int R>
    __device__ __forceinline__ uint32_t seen4(const State &st, int t) const
    {
        const int i = st.qi[R], j = t - prefix;
        uint32_t s;
        if (!a.mask) {
            s = (16u >> (3 - max(-1, min(i - j, 3)))) - 1;   // the lowest i - j + 1 bits
        } else if (a.words == 1) {
            const int up = max(0, min(-j, 4));   // older tokens among the four
            s = (uint32_t)(st.word[R] >> max(0, min(j, 63))) << up | ((1u << up) - 1);
            if (j > 63) s = 0;
        } else {
            s = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) s |= (t + k < len && sees(i, j + k) ? 1u : 0u) << k;
        }
        return s & ((1u << max(0, min(len - t, 4))) - 1);
    }

    // References move only when a score exceeds the last maximum that they were taken from by
    // more than 8; in half precision they stand 2^7 below it, so that weights that vanish are
    // below 2^-32 of the row's largest.
    static constexpr float kBelow = MT == KVR_DT_FP16 ? 7.0f : 0.0f;

    __device__ __forceinline__ bool compute(int step, const char *tile, State &st) const
    {
        f32x4 sc[RT][2];
        static_for<0, 2 * RT>([&](auto I) {
            sc[decltype(I)::value / 2][decltype(I)::value % 2] = f32x4{0, 0, 0, 0};
        });
        static_for<0, NB>([&](auto I) {
            constexpr int i = decltype(I)::value;
            static_for<0, 2>([&](auto T) {
                constexpr int t = decltype(T)::value;
                const char *p = i < RK ? tile + key_at[i & 3] + (i >> 2) * 256 + t * 16 * Rank * 2
                                       : tile + tail_at[i < RK ? 0 : i - RK] + t * 16 * 64 * RO;
                const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
                static_for<0, RT>([&](auto R) {
                    constexpr int r = decltype(R)::value;
                    sc[r][t] = mfma<MT>(x, st.q[r][i], sc[r][t]);
                });
            });
        });
        const bool hides = (step + 1) * kStep > prefix;
        if (hides) {
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const int t = token(step, 0);
                const uint32_t seen = seen4<r>(st, t) | seen4<r>(st, t + 16) << 4;
                const f32x4 x = sc[r][0], y = sc[r][1];
                auto pick = [&](int i, float z) { return seen >> i & 1 ? z : -INFINITY; };
                sc[r][0] = f32x4{pick(0, x[0]), pick(1, x[1]), pick(2, x[2]), pick(3, x[3])};
                sc[r][1] = f32x4{pick(4, y[0]), pick(5, y[1]), pick(6, y[2]), pick(7, y[3])};
            });
        }
        float top[RT];
        bool moves = false;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const f32x4 x = sc[r][0], y = sc[r][1];
            top[r] = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                           fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))) * a.scale2;
            moves = moves || top[r] > st.m[r] + (8.0f + kBelow);
        });
        if (__ballot(moves)) {
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const float t = fmaxf(row_max(top[r]) - kBelow, st.m[r]);
                const float f = __builtin_amdgcn_exp2f(st.m[r] - t);
                st.l[r] *= f;
                st.w[r] *= f;
                static_for<0, 2 * RK>([&](auto E) { st.o[r][decltype(E)::value] *= f; });
                st.m[r] = t;
            });
        }
        u32x4 pv[RT];
        constexpr uint32_t one = MT == KVR_DT_BF16 ? 0x3f803f80u : 0x3c003c00u;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const f32x4 s0 = sc[r][0], s1 = sc[r][1];
            float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -st.m[r]));
            st.l[r] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
            for (int i = 0; i < 4; ++i) pv[r][i] = pack16<MT>(x[2 * i], x[2 * i + 1]);
            // the outputs are divided by the sum of the weights as rounded
            st.w[r] = mfma<MT>(u32x4{one, one, one, one}, pv[r], st.w[r]);
        });
        bool odd = false;
        static_for<0, 2 * RK>([&](auto E) {
            constexpr int e = decltype(E)::value;
            const char *p = tile + val_at[e & 7] + (e >> 3) * 256;
            const u32x2 lo = read_across(p), hi = read_across(p + 16 * Rank * 2);
            uint32_t w[4] = {lo[0], lo[1], hi[0], hi[1]};
            if (hides) {   // a weight of zero would not hide an infinity or a NaN: add_odd puts
                           // them back for the rows that see them
#pragma unroll
                for (int i = 0; i < 4; ++i) odd |= clear_odd2<MT>(w[i]);
            }
            const u32x4 x = {w[0], w[1], w[2], w[3]};
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                st.o[r][e] = mfma<MT>(x, pv[r], st.o[r][e]);
            });
        });
        return odd;
    }

    // ---- infinities and NaN in steps where some tokens are hidden ------------------------

    // Whether element d of token t's latent is one.
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
    // What compute() took out, to four elements from d on of one row.  The same element was part of
    // the score: that is an infinity or a NaN too, the weight 0 or NaN, and their product NaN.
    __device__ __forceinline__ void add_odd(const Part &p, int row, int d, float *x) const
    {
        const int i = row / a.group;
        const int t1 = min(len, p.last * kStep);
        for (int t = max(p.first, prefix / kStep) * kStep; t < t1; ++t) {
            if (!sees(i, t - prefix)) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (odd_at(t, d + e)) x[e] = __uint_as_float(0x7fc00000u);
        }
    }

    // ---- the block -----------------------------------------------------------------------

    // Queries from row r0 on; rows past the last repeat it.
    __device__ __forceinline__ void load_queries(int r0, int rows, State &st) const
    {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = min(r0 + 16 * r + n, rows - 1);
            st.qi[r] = row / a.group;
            const int head = row - st.qi[r] * a.group;
            st.word[r] = a.mask && a.words == 1 ? a.mask[q0 + st.qi[r]] : 0;
            const char *src = a.q.p + ((int64_t)(q0 + st.qi[r]) * a.q.token_stride +
                                       (int64_t)head * a.q.head_stride) * 2;
            const uint32_t flip = a.negate ? 0x80008000u : 0u;
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value;
                st.q[r][i] = *reinterpret_cast<const u32x4 *>(src + (i * 32 + g * 8) * 2) ^ flip;
            });
            st.m[r] = kLowest;
            st.l[r] = 0.0f;
            st.w[r] = f32x4{0, 0, 0, 0};
            static_for<0, 2 * RK>([&](auto E) { st.o[r][decltype(E)::value] = f32x4{0, 0, 0, 0}; });
        }
    }

    // Four elements from d on of a row of the output, or of a part's.
    __device__ __forceinline__ void store(const Part &p, int r0, int row, int d, const float *x,
                                          float top, float sum, float norm) const
    {
        if (p.parts != 1) {
            const int64_t cell = (int64_t)blockIdx.x * BlockRows + row;
            *reinterpret_cast<f32x4 *>(a.part_o + cell * Rank + d) = f32x4{x[0], x[1], x[2], x[3]};
            if (d == 0) a.part_ml[cell] = float4{top, sum, norm, 0.0f};
            return;
        }
        const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
        const int i0 = (r0 + row) / a.group;
        const int head = r0 + row - i0 * a.group;
        char *y = a.out.p + ((int64_t)(q0 + i0) * a.out.token_stride + (int64_t)head * a.out.head_stride + d) * 2;
        *reinterpret_cast<u32x2 *>(y) = u32x2{pack16<MT>(x[0] * inv, x[1] * inv),
                                              pack16<MT>(x[2] * inv, x[3] * inv)};
        if (d == 0 && a.lse)
            a.lse[(int64_t)(q0 + i0) * a.q_heads + head] =
                sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }

    __device__ __forceinline__ void run(char *lds)
    {
        const Part p = find_part(a, (int)blockIdx.x);
        if (p.b < 0) return;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int group = wave / WR, part = wave % WR;
        const int rows = p.nq * a.group, r0 = p.rb * BlockRows;
        len = p.len;
        prefix = p.len - p.nq;
        q0 = p.q0;
        pages = a.pages + (int64_t)p.b * a.pages_stride;
        State st;
        const int w0 = 16 * RT * part;
        load_queries(r0 + w0, rows, st);
        char *tile = lds + group * Buffers * Tile;
        bool odd = false;
        if constexpr (WR == 1) {
            for (int s = p.first + group; s < p.last; s += WT) {
                const Where w = locate(s);
                asm volatile("" ::: "memory");   // the tile has been read
                if constexpr (Quant) {
                    Codes c;
                    fetch_codes(w, 0, c);
                    put_codes(c, 0, tile);
                } else {
                    fetch(w, 0, tile);
                    wait_loads();
                }
                odd |= compute(s, tile, st);
            }
        } else {
            const int rounds = (p.last - p.first + WT - 1) / WT;
            const bool active = r0 + w0 < rows;
            if constexpr (Quant) {
                for (int k = 0; k < rounds; ++k) {
                    const int s = p.first + k * WT + group;
                    if (s < p.last) {
                        Codes c;
                        fetch_codes(locate(s), part, c);
                        put_codes(c, part, tile);
                    }
                    __syncthreads();
                    if (s < p.last && active) odd |= compute(s, tile, st);
                    __syncthreads();
                }
            } else {
                if (p.first + group < p.last) fetch(locate(p.first + group), part, tile);
                for (int k = 0; k < rounds; ++k) {
                    const int s = p.first + k * WT + group;
                    wait_loads();
                    __syncthreads();   // the step's rows are there, the other buffer has been read
                    if (s + WT < p.last) fetch(locate(s + WT), part, tile + ((k + 1) & 1) * Tile);
                    if (s < p.last && active) odd |= compute(s, tile + (k & 1) * Tile, st);
                }
            }
        }
        odd = __syncthreads_or(odd);
        if constexpr (WT == 1) {
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const int row = w0 + 16 * r + n;
                const float sum = row_sum(st.l[r]);
                if (r0 + row >= rows) return;
                static_for<0, 2 * RK>([&](auto E) {
                    constexpr int e = decltype(E)::value;
                    float x[4] = {st.o[r][e][0], st.o[r][e][1], st.o[r][e][2], st.o[r][e][3]};
                    const int d = 16 * e + 4 * g;
                    if (odd) add_odd(p, r0 + row, d, x);
                    store(p, r0, row, d, x, st.m[r], sum, st.w[r][0]);
                });
            });
        } else {
            // Join the groups: maxima first, then values and sums in their order.
            float *sm = reinterpret_cast<float *>(lds + LdsBytes - StatBytes);
            float *sl = sm + Waves * 16 * RT, *sw = sl + Waves * 16 * RT;
            float *so = reinterpret_cast<float *>(lds);
            const int mine = wave * 16 * RT;
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const float sum = row_sum(st.l[r]);
                if (g == 0) {
                    sm[mine + 16 * r + n] = st.m[r];
                    sl[mine + 16 * r + n] = sum;
                    sw[mine + 16 * r + n] = st.w[r][0];
                }
            });
            __syncthreads();
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                float top = kLowest;
#pragma unroll
                for (int t = 0; t < WT; ++t) top = fmaxf(top, sm[(t * WR + part) * 16 * RT + 16 * r + n]);
                const float f = __builtin_amdgcn_exp2f(st.m[r] - top);
                float *row = so + (wave * 16 + n) * JoinRow;
                static_for<0, 2 * RK>([&](auto E) {
                    constexpr int e = decltype(E)::value;
                    *reinterpret_cast<f32x4 *>(row + 16 * e + 4 * g) = st.o[r][e] * f;
                });
                __syncthreads();
                for (int i = threadIdx.x; i < 16 * WR * (Rank / 4); i += 64 * Waves) {
                    const int of = i / (Rank / 4), d = 4 * (i - of * (Rank / 4));   // of: part * 16 + row
                    const int row_at = 16 * RT * (of >> 4) + 16 * r + (of & 15);
                    if (r0 + row_at >= rows) continue;
                    float mx = kLowest, sum = 0.0f, norm = 0.0f;
#pragma unroll
                    for (int t = 0; t < WT; ++t)
                        mx = fmaxf(mx, sm[(t * WR + (of >> 4)) * 16 * RT + 16 * r + (of & 15)]);
                    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < WT; ++t) {
                        const int at = (t * WR + (of >> 4)) * 16 * RT + 16 * r + (of & 15);
                        const float h = __builtin_amdgcn_exp2f(sm[at] - mx);
                        sum += sl[at] * h;
                        norm += sw[at] * h;
                        acc += *reinterpret_cast<const f32x4 *>(
                            so + ((t * WR + (of >> 4)) * 16 + (of & 15)) * JoinRow + d);
                    }
                    float x[4] = {acc[0], acc[1], acc[2], acc[3]};
                    if (odd) add_odd(p, r0 + row_at, d, x);
                    store(p, r0, row_at, d, x, mx, sum, norm);
                }
                if (r + 1 < RT) __syncthreads();
            });
        }
    }
};

template <int FMT, int RK, int RO, int RT, int WR>
__global__ __launch_bounds__(256, 1) void latent_kernel(LatentAttention l)
{
    using K = LatentKernel<FMT, RK, RO, RT, WR>;
    __shared__ __align__(1024) char lds[K::LdsBytes];
    K k(l);
    k.run(lds);
}

template <int FMT, int RK, int RO, int RT, int WR>
hipError_t launch_latent_kernel(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    if (l.a.block_rows != LatentKernel<FMT, RK, RO, RT, WR>::BlockRows) return hipErrorInvalidValue;
    latent_kernel<FMT, RK, RO, RT, WR><<<grid, 256, 0, stream>>>(l);
    return hipGetLastError();
}

template <int FMT, int RK, int RO>
hipError_t launch_latent_rows(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    switch (l.a.block_rows) {   // as plan_latent_attention chose
    case 16: return launch_latent_kernel<FMT, RK, RO, 1, 1>(l, grid, stream);
    case 32: return launch_latent_kernel<FMT, RK, RO, 2, 1>(l, grid, stream);
    case 64: return launch_latent_kernel<FMT, RK, RO, 2, 2>(l, grid, stream);
    default: return launch_latent_kernel<FMT, RK, RO, 2, 4>(l, grid, stream);
    }
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
