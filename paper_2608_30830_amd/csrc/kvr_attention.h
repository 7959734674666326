// Attention of one or more new (drafted) tokens of each sequence over its pages
// of the cache:
//   out_r = sum_j p_rj v_j / sum_j p_rj,   p_rj = exp(scale q_r . k_j - m_r),
// one pass over the cached tokens with the running maximum m_r and sum.  A row r
// is one query head of one new token; the rows of all query heads that share a
// KV head are worked on together, so the cache is read once for them.
//
// Matrix instructions compute S^T = K Q^T and O^T = V^T P^T (16x16x32), with
// cached tokens along the rows of S^T.  Then every lane owns one row r (lane
// mod 16): its scores, its running maximum and its part of O^T, so the softmax
// needs no layout change and P^T leaves the first product in the layout that
// the second one takes (the order of tokens inside a step is free, as long as V
// uses the same).  Keys go from memory to the matrix instruction as they lie.
// Of the values a lane loads eight tokens x eight adjacent elements and turns
// that block around in registers (one byte permute for two elements).  Codes
// become bfloat16 by the format conversions, which apply the block's power of
// two on the way and are exact.
//
// Each wave takes every n-th step of 32 tokens and keeps the loads of the next
// steps in flight; a block joins its waves through LDS.  The sequences are cut
// along the cached tokens into about as many equal parts as fill the GPU (from
// the lengths, on the device); combine_kernel joins the parts.
//
// Each source that includes this header builds the kernel for one cache format
// and query type.
#pragma once

#include <type_traits>

#include "kvr_parts.h"

namespace kvr {
namespace kv {
namespace {

// Every wave computes the same: the parts of all sequences, and where `item` falls.
__device__ Part find_part(const Attention &a, int item)
{
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int len = 0, nq = 0, q0;
        if (b0 + lane < a.n_seqs) sequence(a, b0 + lane, len, nq, q0);
        total += wave_sum(steps_of(len, nq));
    }
    const int per = part_steps(a, total);
    int base = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int len = 0, nq = 0, q0 = 0;
        if (b0 + lane < a.n_seqs) sequence(a, b0 + lane, len, nq, q0);
        const int steps = steps_of(len, nq);
        const int parts = (steps + per - 1) / per;
        const int upto = wave_scan(parts);
        const uint64_t hit = __ballot(base + upto > item);
        if (hit) {
            const int w = __ffsll((unsigned long long)hit) - 1;
            Part p;
            p.b = b0 + w;
            p.parts = lane_value(parts, w);
            p.base = base + lane_value(upto, w) - p.parts;
            p.part = item - p.base;
            p.len = lane_value(len, w);
            p.nq = lane_value(nq, w);
            p.q0 = lane_value(q0, w);
            const int s = lane_value(steps, w);
            p.first = (int)((int64_t)s * p.part / p.parts);
            p.last = (int)((int64_t)s * (p.part + 1) / p.parts);
            return p;
        }
        base += lane_value(upto, 63);
    }
    Part none{};
    none.b = -1;
    return none;
}

// ---- tiles in registers -----------------------------------------------------------

template <int FMT>
struct Fmt {   // bytes of eight elements, and 32-element steps of a key slab of 16-byte loads
    static constexpr int B8 = FMT == KVR_KV_FP8 ? 8 : FMT == KVR_KV_FP4 ? 4 : 16;
    static constexpr int KS = FMT == KVR_KV_FP8 ? 2 : FMT == KVR_KV_FP4 ? 4 : 1;
    static constexpr bool Quant = FMT == KVR_KV_FP8 || FMT == KVR_KV_FP4;
};

template <int I, int N, class F>
__device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// B bytes (1, 2, 4, 8 or 16) from p into words.
template <int B>
__device__ __forceinline__ void load_words(const char *p, uint32_t *w)
{
    if (B == 16) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
        w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
    } else if (B == 8) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
        w[0] = x[0], w[1] = x[1];
    } else if (B == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
    } else if (B == 2) {
        w[0] = *reinterpret_cast<const uint16_t *>(p);
    } else {
        w[0] = *reinterpret_cast<const uint8_t *>(p);
    }
}

// One tile of 16 keys: this lane's token, its chunk of every slab.  A slab is 1, 2
// or 4 blocks of 32 elements, so wide that a lane's chunk of it (a quarter) is 16
// bytes where the head dimension allows.
template <int FMT, int NB>
struct KeyRaw {
    static constexpr int width(int s)   // blocks of slab s
    {
        int start = 0;
        for (;; --s) {
            int w = Fmt<FMT>::KS;
            while (w > NB - start) w >>= 1;
            if (s == 0) return w;
            start += w;
        }
    }
    static constexpr int start(int s) { return s == 0 ? 0 : start(s - 1) + width(s - 1); }
    static constexpr int count()
    {
        int n = 0;
        while (start(n) < NB) ++n;
        return n;
    }
    static constexpr int slabs = count();
    static constexpr int slab_of(int block)
    {
        int s = 0;
        while (start(s) + width(s) <= block) ++s;
        return s;
    }
    uint32_t w[NB * Fmt<FMT>::B8 / 4];
    uint32_t s[Fmt<FMT>::Quant ? slabs : 1];   // scale byte of each chunk
};
// One step of values: this lane's chunk of its eight tokens in every slab.  A slab
// is 16 lanes of 8, 4 or 2 elements.
template <int FMT, int NB>
struct ValRaw {
    static constexpr int wide = NB / 4, mid = (NB & 2) ? 1 : 0, low = NB & 1;
    static constexpr int slabs = wide + mid + low;
    static constexpr int width(int s) { return s < wide ? 8 : s == wide && mid ? 4 : 2; }
    static constexpr int first(int s) { return s == 0 ? 0 : first(s - 1) + width(s - 1); }
    static constexpr int word(int s)
    {
        return s == 0 ? 0 : word(s - 1) + (Fmt<FMT>::B8 * width(s - 1) / 8 + 3) / 4;
    }
    static constexpr int slab_of(int e)
    {
        int s = 0;
        while (first(s) + width(s) <= e) ++s;
        return s;
    }
    static constexpr int words = word(slabs);
    uint32_t w[8][words];
    uint32_t s[8][Fmt<FMT>::Quant ? slabs : 1];
};

// ---- the kernel -------------------------------------------------------------------

template <int QT>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if (QT == KVR_DT_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Largest / sum over the four lanes (16 apart) that share a row.
__device__ __forceinline__ float row_max(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row_sum(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel)
{
    return __builtin_amdgcn_perm(hi, lo, sel);
}

template <int FMT, int QT, int NB, int RT, int PF>
struct Kernel {
    static constexpr int D = NB * 32;
    static constexpr bool Quant = Fmt<FMT>::Quant;
    static constexpr int MT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // product type
    // a half-precision query against a quantised cache is split into two bfloat16 parts
    static constexpr int QS = Quant && QT == KVR_DT_FP16 ? 2 : 1;
    static constexpr int Rows16 = 16 * RT;
    static constexpr int LdsRow = D + 4;
    using KR = KeyRaw<FMT, NB>;
    using VR = ValRaw<FMT, NB>;

    struct Stage {
        KR k[2];
        VR v;
    };

    const Attention &a;
    const uint32_t n, g;
    int h, len, prefix;
    const int32_t *pages;
    uint32_t krow, vrow, ksrow, vsrow;   // byte offsets of this lane's rows in a tile

    __device__ Kernel(const Attention &a_)
        : a(a_), n(threadIdx.x & 15), g((threadIdx.x & 63) >> 4)
    {
        krow = (uint32_t)n * (uint32_t)a.c.token_stride;
        vrow = 4u * (uint32_t)g * (uint32_t)a.c.token_stride;
        ksrow = (uint32_t)n * (uint32_t)a.c.stoken_stride;
        vsrow = 4u * (uint32_t)g * (uint32_t)a.c.stoken_stride;
    }

    // The page and the first row in it of the 16 tokens from t on (any tile that
    // begins at or past the sequence's end is read as its last tile).
    __device__ __forceinline__ void tile_at(int t, int64_t &page, int &off) const
    {
        const int last = (len - 1) & ~15;
        t = t < last ? t : last;
        int id = pages[t >> a.c.page_shift];
        id = __builtin_amdgcn_readfirstlane(id);
        if (id < 0 || id >= a.c.n_pages) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            id = 0;
        }
        page = id;
        off = t & ((1 << a.c.page_shift) - 1);
    }

    __device__ __forceinline__ void load(int step, Stage &st) const
    {
        // Uniform addresses plus one 32-bit lane offset for all keys, one for all values.
        const int64_t ts = a.c.token_stride, sts = a.c.stoken_stride;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            int64_t page;
            int off;
            tile_at(step * kStep + 16 * t, page, off);
            const int64_t at = page * a.c.page_stride + h * a.c.head_stride + off * ts;
            const char *kp = a.c.k + at, *vp = a.c.v + at;
            const uint8_t *ksp = nullptr, *vsp = nullptr;
            if (Quant) {
                const int64_t sat = page * a.c.spage_stride + h * a.c.shead_stride + off * sts;
                ksp = a.c.ks + sat;
                vsp = a.c.vs + sat;
            }
            // keys: token n of the tile, chunk g of every slab
            static_for<0, KR::slabs>([&](auto S) {
                constexpr int s = decltype(S)::value;
                constexpr int start = KR::start(s), width = KR::width(s), B8 = Fmt<FMT>::B8;
                load_words<width * B8>(kp + start * 4 * B8 + (krow + g * (width * B8)),
                                       &st.k[t].w[start * B8 / 4]);
                if constexpr (Quant)
                    st.k[t].s[s] = (ksp + start)[ksrow + (uint32_t)(g * width / 4)];
            });
            // values: tokens 4 g + j of the tile, chunk n of every slab
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                static_for<0, VR::slabs>([&](auto S) {
                    constexpr int s = decltype(S)::value;
                    constexpr int W = VR::width(s), B = Fmt<FMT>::B8 * W / 8;
                    constexpr int e0 = VR::first(s);   // elements / 16 before the slab
                    load_words<B>(vp + j * ts + e0 * 16 * Fmt<FMT>::B8 / 8 + (vrow + n * B),
                                  &st.v.w[4 * t + j][VR::word(s)]);
                    if constexpr (Quant)
                        st.v.s[4 * t + j][s] =
                            (vsp + j * sts + e0 / 2)[vsrow + (uint32_t)(n * W / 32)];
                });
            }
        }
    }

    // Block I of a key tile as the matrix instruction takes it: eight elements.
    template <int I>
    __device__ __forceinline__ u32x4 key_block(const KR &k) const
    {
        if constexpr (!Quant) {
            return u32x4{k.w[4 * I], k.w[4 * I + 1], k.w[4 * I + 2], k.w[4 * I + 3]};
        } else {
            constexpr int slab = KR::slab_of(I);
            const float s = scale_of(k.s[slab]);
            if constexpr (FMT == KVR_KV_FP8)
                return u32x4{codes_to_bf16x2<FMT, 0>(k.w[2 * I], s),
                             codes_to_bf16x2<FMT, 1>(k.w[2 * I], s),
                             codes_to_bf16x2<FMT, 0>(k.w[2 * I + 1], s),
                             codes_to_bf16x2<FMT, 1>(k.w[2 * I + 1], s)};
            else
                return u32x4{codes_to_bf16x2<FMT, 0>(k.w[I], s), codes_to_bf16x2<FMT, 1>(k.w[I], s),
                             codes_to_bf16x2<FMT, 2>(k.w[I], s), codes_to_bf16x2<FMT, 3>(k.w[I], s)};
        }
    }

    // Elements 2 I, 2 I + 1 (over all slabs) of one token's chunks as 16-bit values.
    template <int I>
    __device__ __forceinline__ uint32_t val_pair(const VR &v, int tok) const
    {
        constexpr int s = VR::slab_of(2 * I), i = I - VR::first(s) / 2, w = VR::word(s);
        if constexpr (!Quant) return v.w[tok][w + i];
        else {
            const float sc = scale_of(v.s[tok][s]);
            if constexpr (FMT == KVR_KV_FP8)
                return codes_to_bf16x2<FMT, i & 1>(v.w[tok][w + i / 2], sc);
            else return codes_to_bf16x2<FMT, i>(v.w[tok][w], sc);
        }
    }

    __device__ __forceinline__ static bool nonfinite(uint32_t x)
    {
        constexpr uint32_t e = MT == KVR_DT_BF16 ? 0x7f80u : 0x7c00u;
        return (x & e) == e || (x & (e << 16)) == (e << 16);
    }

    // Non-finite halves of x to zero, and what they were: 1 (NaN), 64 (+inf) or 4096 (-inf).
    __device__ __forceinline__ static void split(uint32_t &x, uint32_t &flag)
    {
        constexpr uint32_t e = MT == KVR_DT_BF16 ? 0x7f80u : 0x7c00u;
        flag = 0;
        uint32_t kept = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t y = (x >> (16 * i)) & 0xffffu;
            float f = 0.0f;
            if ((y & e) == e) f = (y & 0x7fffu) != e ? 1.0f : (y & 0x8000u) ? 4096.0f : 64.0f;
            else kept |= y << (16 * i);
            flag |= (pack16<MT>(f, 0.0f) & 0xffffu) << (16 * i);
        }
        x = kept;
    }

    // One step: scores of 32 tokens, softmax update, values.
    __device__ __forceinline__ void compute(int step, Stage &st, const u32x4 (&q)[RT][QS][NB],
                                            f32x4 (&o)[RT][2 * NB], float (&m)[RT], float (&l)[RT],
                                            const int (&qi)[RT], int q0, int nq) const
    {
        const int t0 = step * kStep;
        f32x4 sc[RT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int r = 0; r < RT; ++r) sc[r][t] = f32x4{0, 0, 0, 0};
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value;
                const u32x4 kb = key_block<i>(st.k[t]);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int p = 0; p < QS; ++p) sc[r][t] = mfma<MT>(kb, q[r][p][i], sc[r][t]);
            });
        }
        const bool masked = t0 + kStep > prefix;
        const bool ends = t0 + kStep > len;
        u32x4 pv[RT], vis[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float x[8];
            uint32_t seen = 0xff;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = sc[r][i >> 2][i & 3] * a.scale2;
            if (masked) {
                seen = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = t0 + 16 * (i >> 2) + 4 * (int)g + (i & 3);
                    const int j = t - prefix;
                    bool v = j < 0;
                    if (!v && t < len) {
                        if (a.mask)
                            v = (a.mask[(int64_t)(q0 + qi[r]) * a.words + (j >> 6)] >> (j & 63)) & 1;
                        else v = j <= qi[r];
                    }
                    x[i] = v ? x[i] : -INFINITY;
                    seen |= (v ? 1u : 0u) << i;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                              fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            top = fmaxf(row_max(top), m[r]);
            if (__ballot(top > m[r])) {
                const float f = __builtin_amdgcn_exp2f(m[r] - top);
                l[r] *= f;
#pragma unroll
                for (int e = 0; e < 2 * NB; ++e) o[r][e] *= f;
                m[r] = top;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = __builtin_amdgcn_exp2f(x[i] - m[r]);
                l[r] += x[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pv[r][i] = pack16<MT>(x[2 * i], x[2 * i + 1]);
                vis[r][i] = masked ? pack16<MT>(seen >> (2 * i) & 1, seen >> (2 * i + 1) & 1) : 0u;
            }
        }
        if (ends) {   // rows past the end hold anything: they read as zeros
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + 16 * (i >> 2) + 4 * (int)g + (i & 3) >= len) {
#pragma unroll
                    for (int w = 0; w < VR::words; ++w) st.v.w[i][w] = 0;
                    if (Quant)
#pragma unroll
                        for (int s = 0; s < VR::slabs; ++s) st.v.s[i][s] = 127;
                }
        }
        bool odd = false;
        if (masked) {   // may a hidden token hold an infinity or a NaN?
            static_for<0, NB>([&](auto I) {
#pragma unroll
                for (int t = 0; t < 8; ++t) odd = odd || nonfinite(val_pair<decltype(I)::value>(st.v, t));
            });
        }
        if (__ballot(odd)) values<true>(st.v, pv, vis, o);
        else values<false>(st.v, pv, vis, o);
    }

    // O^T += V^T P^T.  Odd: the non-finite values are taken out and counted apart, for
    // the rows that see their tokens.
    template <bool Odd>
    __device__ __forceinline__ void values(const VR &v, const u32x4 (&pv)[RT], const u32x4 (&vis)[RT],
                                           f32x4 (&o)[RT][2 * NB]) const
    {
        static_for<0, NB>([&](auto I) {
            constexpr int i = decltype(I)::value;   // elements 2 i and 2 i + 1 of the chunks
            uint32_t c[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) c[t] = val_pair<i>(v, t);
            u32x4 x[2];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[0][t] = perm(c[2 * t + 1], c[2 * t], 0x05040100u);
                x[1][t] = perm(c[2 * t + 1], c[2 * t], 0x07060302u);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                u32x4 flags;
                if (Odd) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        uint32_t y = x[e][t], f;
                        split(y, f);
                        x[e][t] = y;
                        flags[t] = f;
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if (Odd) {
                        const f32x4 f = mfma<MT>(flags, vis[r], f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int bits = (int)f[k];
                            float add = 0.0f;
                            if ((bits & 63) || ((bits & 4032) && bits >= 4096))
                                add = __uint_as_float(0x7fc00000u);
                            else if (bits >= 4096) add = -INFINITY;
                            else if (bits) add = INFINITY;
                            o[r][2 * i + e][k] += add;
                        }
                    }
                    o[r][2 * i + e] = mfma<MT>(x[e], pv[r], o[r][2 * i + e]);
                }
            }
        });
    }

    __device__ __forceinline__ void run(float *lds)
    {
        // The row blocks of one part share its cached tokens: they go to one XCD
        // (block number mod 8), one after another.
        const int rb8 = 8 * a.row_blocks;
        const int grp = blockIdx.x / rb8, in = blockIdx.x - grp * rb8;
        const int rb = in >> 3;
        const int unit = grp * 8 + (in & 7);
        const int nh = a.c.n_heads;
        const int item = unit / nh;
        h = unit - item * nh;
        const Part p = find_part(a, item);
        if (p.b < 0) return;
        const int rows = p.nq * a.group;
        const int r0 = rb * Rows16;
        if (r0 >= rows) return;
        len = p.len;
        prefix = p.len - p.nq;
        pages = a.pages + (int64_t)p.b * a.pages_stride;

        u32x4 q[RT][QS][NB];
        f32x4 o[RT][2 * NB];
        float m[RT], l[RT];
        int qi[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = min(r0 + 16 * r + (int)n, rows - 1);   // rows past the last repeat it
            qi[r] = row / a.group;
            const int head = h * a.group + (row - qi[r] * a.group);
            const char *src = a.q.p + ((int64_t)(p.q0 + qi[r]) * a.q.token_stride +
                                       (int64_t)head * a.q.head_stride) * 2;
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value, s = KR::slab_of(i), start = KR::start(s);
                const int d = start * 32 + g * KR::width(s) * 8 + (i - start) * 8;
                u32x4 x = *reinterpret_cast<const u32x4 *>(src + d * 2);
                if (QS == 2) {
                    u32x4 lo;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        float x0, x1, y0, y1;
                        unpack16<KVR_DT_FP16>(x[t], x0, x1);
                        x[t] = pack_bf16(x0, x1);
                        unpack16<KVR_DT_BF16>(x[t], y0, y1);
                        lo[t] = pack_bf16(x0 - y0, x1 - y1);
                    }
                    q[r][QS - 1][i] = lo;
                }
                q[r][0][i] = x;
            });
            m[r] = kLowest;
            l[r] = 0.0f;
#pragma unroll
            for (int e = 0; e < 2 * NB; ++e) o[r][e] = f32x4{0, 0, 0, 0};
        }

        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        Stage st[PF];
        int s = p.first + wave;
#pragma unroll
        for (int i = 0; i < PF; ++i)
            if (s + i * kWaves < p.last) load(s + i * kWaves, st[i]);
        for (; s < p.last; s += PF * kWaves) {
#pragma unroll
            for (int i = 0; i < PF; ++i) {
                const int at = s + i * kWaves;
                if (at < p.last) {
                    compute(at, st[i], q, o, m, l, qi, p.q0, p.nq);
                    if (at + PF * kWaves < p.last) load(at + PF * kWaves, st[i]);
                }
            }
        }

        // join the waves: maxima first, then sums and values in wave order
        float *sm = lds, *sl = lds + kWaves * Rows16, *so = lds + 2 * kWaves * Rows16;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            l[r] = row_sum(l[r]);
            if (g == 0) {
                sm[wave * Rows16 + 16 * r + n] = m[r];
                sl[wave * Rows16 + 16 * r + n] = l[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = kLowest;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w * Rows16 + 16 * r + n]);
            const float f = __builtin_amdgcn_exp2f(m[r] - top);
#pragma unroll
            for (int e = 0; e < 2 * NB; ++e) o[r][e] *= f;
        }
        for (int w = 0; w < kWaves; ++w) {
            if (wave == w) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    float *row = so + (16 * r + n) * LdsRow;
static_for<0, 2 * NB>([&](auto E) {
                        // tile e of its slab: element (4 g + i) * W + e - e0 of the slab
                        constexpr int e = decltype(E)::value, slab = VR::slab_of(e);
                        constexpr int e0 = VR::first(slab), W = VR::width(slab);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float *x = row + 16 * e0 + (4 * g + i) * W + (e - e0);
                            *x = w == 0 ? o[r][e][i] : *x + o[r][e][i];
                        }
                    });
                }
            }
            __syncthreads();
        }

        // rows out: eight elements a thread
        const bool whole = p.parts == 1;
        const int64_t cell = ((int64_t)(p.base + p.part) * nh + h) * a.row_blocks + rb;
        for (int i = threadIdx.x; i < Rows16 * (D / 8); i += kThreads) {
            const int row = i / (D / 8), d = 8 * (i - row * (D / 8));
            if (r0 + row >= rows) break;
            float top = kLowest, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w * Rows16 + row]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                sum += sl[w * Rows16 + row] * __builtin_amdgcn_exp2f(sm[w * Rows16 + row] - top);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = so[row * LdsRow + d + e];
            if (!whole) {
                store8<KVR_DT_FP32>(
                    reinterpret_cast<char *>(a.part_o + (cell * Rows16 + row) * D + d), x);
                if (d == 0) {
                    a.part_ml[(cell * Rows16 + row) * 2] = top;
                    a.part_ml[(cell * Rows16 + row) * 2 + 1] = sum;
                }
                continue;
            }
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= inv;
            const int i0 = (r0 + row) / a.group;
            const int head = h * a.group + (r0 + row - i0 * a.group);
            store8<QT>(a.out.p + ((int64_t)(p.q0 + i0) * a.out.token_stride +
                                  (int64_t)head * a.out.head_stride + d) * 2, x);
            if (d == 0 && a.lse)
                a.lse[(int64_t)(p.q0 + i0) * a.q_heads + head] =
                    sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
};

template <int FMT, int QT, int NB, int RT, int PF>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(Attention a)
{
    __shared__ float lds[2 * kWaves * 16 * RT + 16 * RT * (NB * 32 + 4)];
    Kernel<FMT, QT, NB, RT, PF> k(a);
    k.run(lds);
}

// One launch for a format and query type, the head size and the row tiles chosen here.
template <int FMT, int QT, int NB, int RT>
hipError_t launch_rt(const Attention &a, dim3 grid, hipStream_t stream)
{
    constexpr int stage = NB * Fmt<FMT>::B8;   // registers of one step's keys and values
    constexpr int room = (Fmt<FMT>::Quant ? 64 : RT == 1 ? 128 : 64) / stage;
    constexpr int PF = room < 1 ? 1 : room > 3 ? 3 : room;
    attention_kernel<FMT, QT, NB, RT, PF><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int FMT, int QT, int NB>
hipError_t launch_nb(const Attention &a, dim3 grid, hipStream_t stream)
{
    if (a.row_tiles == 1) return launch_rt<FMT, QT, NB, 1>(a, grid, stream);
    return launch_rt<FMT, QT, NB, 2>(a, grid, stream);
}

template <int FMT, int QT>
hipError_t launch_dim(const Attention &a, dim3 grid, hipStream_t stream)
{
    switch (a.c.dim) {
#ifndef KVR_DEV_DIM128
    case 64: return launch_nb<FMT, QT, 2>(a, grid, stream);
    case 96: return launch_nb<FMT, QT, 3>(a, grid, stream);
    case 192: return launch_nb<FMT, QT, 6>(a, grid, stream);
    case 256: return launch_nb<FMT, QT, 8>(a, grid, stream);
#endif
    default: return launch_nb<FMT, QT, 4>(a, grid, stream);
    }
}

}  // namespace
}  // namespace kv
}  // namespace kvr
