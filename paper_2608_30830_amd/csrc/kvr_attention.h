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
// With up to 32 rows every wave has all of them and takes every n-th step of 32
// tokens, with the loads of the next steps in flight and their pages looked up a
// round earlier; a block joins its waves through LDS.  Memory bounds this: 64
// sequences of 8,192 tokens, 8 heads of 128, one new token each: 190 us in 8
// bits (5.8 TB/s of cache), 373 us in 16 (5.8), 117 us in 4 (4.9, where the
// conversions begin to count).  With more rows the waves divide them and share
// the tokens through LDS, converted and turned around once: 16 sequences of
// 16,384 tokens and 512 rows, 16 bits: 0.67 ms, 820 TFLOP/s.  There the matrix
// unit is busy for 40 % of the cycles and the vector unit for 44 % (the softmax: a
// multiply-add, an exponential, a sum and half a packing a score, and 20 instructions for
// the maximum of 16, half of which only quiet NaNs), and with the two
// waves that the registers leave a SIMD their sum is what counts: reading LDS
// further ahead, a second buffer in place of one of the two barriers and the
// weights of one step interleaved with the products of the other by hand changed
// the time by less than the runs differ.
//
// The sequences are cut along the cached tokens into about as many equal parts as
// fill the GPU (from the lengths, on the device); combine_kernel joins the parts.
//
// Each source that includes this header builds the kernel for one cache format
// and query type.
#pragma once

#include <type_traits>

#include "kvr_parts.h"

namespace kvr {
namespace kv {
namespace {

// Where `item` falls: parts of sequences in order, each part's row blocks next to each
// other.  Every wave computes the same.
__device__ __forceinline__ Part find_part(const Attention &a, int item)
{
    if (a.direct) {
        Part p{};
        p.b = item / a.direct;
        p.rb = item - p.b * a.direct;
        p.parts = 1;
        sequence(a, p.b, p.len, p.nq, p.q0);
        p.last = steps_of(p.len, p.nq);
        if (p.last == 0 || p.rb >= row_blocks_of(a, p.nq)) p.b = -1;
        return p;
    }
    Lane x = lane_sequence(a, 0);
    const int per = part_steps(a, x);
    if (a.chosen && item == 0 && threadIdx.x == 0) *a.chosen = per;
    int base = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        if (b0) x = lane_sequence(a, b0);
        const int parts = parts_of(a, x.steps, per);
        const int upto = wave_incl_scan(parts * x.rbs);
        const uint64_t hit = __ballot(base + upto > item);
        if (hit) {
            const int w = __ffsll((unsigned long long)hit) - 1;
            Part p;
            p.b = b0 + w;
            p.parts = lane_value(parts, w);
            const int nrb = lane_value(x.rbs, w);
            const int at = item - (base + lane_value(upto, w) - p.parts * nrb);
            p.part = at / nrb;
            p.rb = at - p.part * nrb;
            p.len = lane_value(x.len, w);
            p.nq = lane_value(x.nq, w);
            p.q0 = lane_value(x.q0, w);
            const int s = lane_value(x.steps, w);
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

template <int FMT, int QT, int NB, int RT, int PF, bool Shared, int Waves>
struct Kernel {
    static constexpr int D = NB * 32;
    static constexpr bool Quant = Fmt<FMT>::Quant;
    static constexpr int MT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // product type
    // Half-precision queries and weights meet a quantised cache as two bfloat16 parts.
    static constexpr int QS = Quant && QT == KVR_DT_FP16 ? 2 : 1;
    static constexpr int BlockRows = (Shared ? Waves : 1) * 16 * RT;
    static constexpr int LdsRow = D + 4;
    using KR = KeyRaw<FMT, NB>;
    using VR = ValRaw<FMT, NB>;

    struct Stage {   // one step as loaded
        KR k[2];
        VR v;
    };
    struct State {   // of this wave's rows
        u32x4 q[RT][QS][NB];
        f32x4 o[RT][2 * NB];
        float m[RT], l[RT];   // reference (log2), this lane's part of the weights' sum
        f32x4 w[RT];          // sum of the rounded weights (every element the same)
        int qi[RT];           // query within the sequence
        uint64_t word[RT];    // its tree mask, where that is one word
    };
    // LDS: the joining of the waves (maxima, sums, values), or one step of each wave in
    // the order that the matrix instructions read: keys [2][NB][64], values [2 NB][64].
    static constexpr int JoinWords = (3 + LdsRow) * Waves * BlockRows;
    static constexpr int StepWords = 4 * NB * 64 * 4;
    static constexpr int Tile = Waves / 2;   // steps that a block brings into LDS at a time
    static constexpr int Pair = 2;           // steps that are worked on together
    static constexpr int LdsWords = Shared ? Tile * StepWords : JoinWords;

    const Attention &a;
    const uint32_t n, g, lane;
    int h, len, prefix, q0;
    const int32_t *pages;
    const int last_page;   // of the table's row
    uint32_t krow, vrow, ksrow, vsrow;   // byte offsets of this lane's rows in a tile

    __device__ Kernel(const Attention &a_)
        : a(a_), n(threadIdx.x & 15), g((threadIdx.x & 63) >> 4), lane(threadIdx.x & 63),
          last_page((int)min(a_.max_pages, (int64_t)INT32_MAX) - 1)
    {
        krow = (uint32_t)n * (uint32_t)a.c.token_stride;
        vrow = 4u * (uint32_t)g * (uint32_t)a.c.token_stride;
        ksrow = (uint32_t)n * (uint32_t)a.c.stoken_stride;
        vsrow = 4u * (uint32_t)g * (uint32_t)a.c.stoken_stride;
    }

    // The pages that hold a step's two tiles, as the table has them: looked up well before
    // the rows are loaded, and whatever the sequence's length (within the table's row).
    struct Pages {
        int id[2];
    };
    __device__ __forceinline__ Pages look_up(int step) const
    {
        const int at = step * kStep;   // below 2^31: at most 2^30 tokens and a few steps
        return Pages{{pages[min(at >> a.c.page_shift, last_page)],
                      pages[min((at + 16) >> a.c.page_shift, last_page)]}};
    }

    // Uniform addresses plus one 32-bit lane offset for all keys, one for all values.
    struct Where {   // a tile in the cache and in its scales
        int64_t at, sat;
    };
    // (A second tile that begins past the sequence's end is read as the first.)
    __device__ __forceinline__ Where locate(int step, int t, const Pages &p) const
    {
        const bool past = step * kStep + 16 * t >= len;
        int page = __builtin_amdgcn_readfirstlane(past ? p.id[0] : p.id[t]);
        if (page < 0 || page >= a.c.n_pages) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            page = 0;
        }
        const int off = (step * kStep + (past ? 0 : 16 * t)) & ((1 << a.c.page_shift) - 1);
        return Where{page * a.c.page_stride + h * a.c.head_stride + off * a.c.token_stride,
                     Quant ? page * a.c.spage_stride + h * a.c.shead_stride +
                                 off * a.c.stoken_stride
                           : 0};
    }
    // Token n of the tile, chunk g of every slab.
    __device__ __forceinline__ void load_keys(const Where &at, KR &k) const
    {
        const char *kp = a.c.k + at.at;
        const uint8_t *ksp = a.c.ks + at.sat;
        static_for<0, KR::slabs>([&](auto S) {
            constexpr int s = decltype(S)::value;
            constexpr int start = KR::start(s), width = KR::width(s), B8 = Fmt<FMT>::B8;
            load_words<width * B8>(kp + start * 4 * B8 + (krow + g * (width * B8)),
                                   &k.w[start * B8 / 4]);
            if constexpr (Quant) k.s[s] = (ksp + start)[ksrow + (uint32_t)(g * width / 4)];
        });
    }
    // Tokens 4 g + j of the tile, chunk n of every slab.
    __device__ __forceinline__ void load_values(const Where &at, int t, VR &v) const
    {
        const int64_t ts = a.c.token_stride, sts = a.c.stoken_stride;
        const char *vp = a.c.v + at.at;
        const uint8_t *vsp = a.c.vs + at.sat;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            static_for<0, VR::slabs>([&](auto S) {
                constexpr int s = decltype(S)::value;
                constexpr int W = VR::width(s), B = Fmt<FMT>::B8 * W / 8;
                constexpr int e0 = VR::first(s);   // elements / 16 before the slab
                load_words<B>(vp + j * ts + e0 * 16 * Fmt<FMT>::B8 / 8 + (vrow + n * B),
                              &v.w[4 * t + j][VR::word(s)]);
                if constexpr (Quant)
                    v.s[4 * t + j][s] = (vsp + j * sts + e0 / 2)[vsrow + (uint32_t)(n * W / 32)];
            });
        }
    }
    __device__ __forceinline__ void load(int step, const Pages &p, Stage &st) const
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const Where at = locate(step, t, p);
            load_keys(at, st.k[t]);
            load_values(at, t, st.v);
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

    // Infinities and NaN among a lane's loaded values, and those values to zero.  A code is odd
    // where its block's scale byte s makes it so: all of them for 255; the two NaN of
    // e4m3; and those whose value reaches 2^128, magnitude bits of (262 - s) * 8 on for e4m3
    // (s >= 247) and (256 - s) * 2 for e2m1 (s >= 253).  That much below a code's top bit is
    // added, so that odd codes carry into it.
    static constexpr uint32_t kExp = FMT == KVR_KV_FP16 ? 0x7c00u : 0x7f80u;
    static constexpr uint32_t kMag = FMT == KVR_KV_FP8 ? 0x7f7f7f7fu : 0x77777777u;
    __device__ __forceinline__ static uint32_t to_odd(uint32_t s)   // of one code
    {
        if (FMT == KVR_KV_FP8) return s < 247 ? 1u : 8u * (s - 246);
        return s < 253 ? 0u : 2u * (s - 252);
    }
    __device__ __forceinline__ static uint32_t odd_codes(uint32_t x, uint32_t s)   // their top bits
    {
        return ((x & kMag) + to_odd(s) * (FMT == KVR_KV_FP8 ? 0x01010101u : 0x11111111u)) & ~kMag;
    }
    __device__ __forceinline__ static bool odd_values(const VR &v)
    {
        bool odd = false;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (!Quant)
#pragma unroll
                for (int w = 0; w < VR::words; ++w) {
                    const uint32_t x = v.w[t][w];
                    odd = odd || (x & kExp) == kExp || (x & kExp << 16) == kExp << 16;
                }
            if constexpr (Quant)
                static_for<0, VR::slabs>([&](auto S) {
                    constexpr int s = decltype(S)::value;
                    odd = odd || v.s[t][s] == kBadScale;
#pragma unroll
                    for (int w = VR::word(s); w < VR::word(s + 1); ++w)
                        odd = odd || odd_codes(v.w[t][w], v.s[t][s]) != 0;
                });
        }
        return __ballot(odd) != 0;
    }
    __device__ __forceinline__ static void clear_odd(VR &v)
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (!Quant)
#pragma unroll
                for (int w = 0; w < VR::words; ++w) {
                    uint32_t x = v.w[t][w];
                    if ((x & kExp) == kExp) x &= 0xffff0000u;
                    if ((x & kExp << 16) == kExp << 16) x &= 0xffffu;
                    v.w[t][w] = x;
                }
            if constexpr (Quant)
                static_for<0, VR::slabs>([&](auto S) {
                    constexpr int s = decltype(S)::value;
                    const bool bad = v.s[t][s] == kBadScale;
#pragma unroll
                    for (int w = VR::word(s); w < VR::word(s + 1); ++w) {
                        const uint32_t top = odd_codes(v.w[t][w], v.s[t][s]);
                        const uint32_t keep = FMT == KVR_KV_FP8 ? ~((top >> 7) * 255u) : ~((top >> 3) * 15u);
                        v.w[t][w] = bad ? 0u : v.w[t][w] & keep;
                    }
                    if (bad) v.s[t][s] = 127;
                });
        }
    }

    // Token i (of this lane's eight) of a step.
    __device__ __forceinline__ int token(int step, int i) const
    {
        return step * kStep + 16 * (i >> 2) + 4 * (int)g + (i & 3);
    }

    // Rows past the sequence's end hold anything: they read as zeros.
    __device__ __forceinline__ void clear_past_end(int step, VR &v) const
    {
        if ((step + 1) * kStep <= len) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (token(step, i) >= len) {
#pragma unroll
                for (int w = 0; w < VR::words; ++w) v.w[i][w] = 0;
                if (Quant)
#pragma unroll
                    for (int s = 0; s < VR::slabs; ++s) v.s[i][s] = 127;
            }
    }

    // A step's values as the products may take them: rows past the end as zeros, and where
    // tokens are hidden from some rows, infinities and NaN as zeros too (a weight of
    // zero would not hide them); add_odd puts them back for the rows that see them.
    __device__ __forceinline__ bool clean(int step, VR &v) const
    {
        if ((step + 1) * kStep <= prefix) return false;   // nothing is hidden
        clear_past_end(step, v);
        const bool odd = odd_values(v);
        if (odd) clear_odd(v);
        return odd;
    }

    // Element d of token t's value, if it is an infinity or a NaN, else 0.
    __device__ __forceinline__ float odd_at(int t, int d) const
    {
        int id = pages[t >> a.c.page_shift];
        if (id < 0 || id >= a.c.n_pages) id = 0;
        const int off = t & ((1 << a.c.page_shift) - 1);
        const char *row = a.c.v + id * a.c.page_stride + h * a.c.head_stride + off * a.c.token_stride;
        if (!Quant) {
            const uint16_t x = reinterpret_cast<const uint16_t *>(row)[d];
            if ((x & kExp) != kExp) return 0.0f;
            return load1<FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16>(row, d);
        }
        const uint32_t sc = a.c.vs[id * a.c.spage_stride + h * a.c.shead_stride +
                                   off * a.c.stoken_stride + (d >> 5)];
        constexpr bool E4 = FMT == KVR_KV_FP8;
        const uint32_t byte = reinterpret_cast<const uint8_t *>(row)[E4 ? d : d >> 1];
        const uint32_t code = E4 ? byte : byte >> 4 * (d & 1) & 15u;
        const uint32_t mag = code & (E4 ? 0x7fu : 7u);
        if (sc == kBadScale || (E4 && mag == 0x7fu)) return __uint_as_float(0x7fc00000u);
        if (mag + to_odd(sc) < (E4 ? 128u : 8u)) return 0.0f;
        return code > mag ? -INFINITY : INFINITY;
    }
    // The infinities and NaN that clean() took out, to W elements of one row.
    template <int W>
    __device__ __forceinline__ void add_odd(const Part &p, int row, int d, float *x) const
    {
        const int i = row / a.group;
        const int t1 = min(len, p.last * kStep);
        for (int t = max(p.first, prefix / kStep) * kStep; t < t1; ++t) {
            if (!sees(i, t - prefix)) continue;
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float y = odd_at(t, d + e);
                if (y != 0.0f) x[e] += y;   // NaN included
            }
        }
    }
    // Whether query i sees newest token j (older ones: j < 0).
    __device__ __forceinline__ bool sees(int i, int j) const
    {
        if (j < 0) return true;
        if (a.mask) return (a.mask[(int64_t)(q0 + i) * a.words + (j >> 6)] >> (j & 63)) & 1;
        return j <= i;
    }

    // The same for tokens t to t + 3 before `end` and the lane's row of tile R, as bits.
    // (A load and a branch for each token and row made short contexts of many rows a third slower.)
    template <int R>
    __device__ __forceinline__ uint32_t seen4(const State &st, int t, int end) const
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
            for (int k = 0; k < 4; ++k) s |= (t + k < end && sees(i, j + k) ? 1u : 0u) << k;
        }
        return s & ((1u << max(0, min(end - t, 4))) - 1);   // of four at most
    }

    // Value tiles 2 I and 2 I + 1 of a step: element pairs of eight tokens turned around.
    template <int I>
    __device__ __forceinline__ void val_tiles(const VR &v, u32x4 (&x)[2]) const
    {
        uint32_t c[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) c[t] = val_pair<I>(v, t);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[0][t] = perm(c[2 * t + 1], c[2 * t], 0x05040100u);
            x[1][t] = perm(c[2 * t + 1], c[2 * t], 0x07060302u);
        }
    }

    // Before the weights of U steps from `step` on (the part ends before step `last`):
    // hidden tokens' scores to -infinity, and the references.  Those move only when a score
    // exceeds the last maximum that they were taken from by more than 8 (weights of up to 2^8
    // lose no precision), so most steps need no exchange between lanes.  In half precision a
    // reference is 2^7 below its maximum: weights reach 2^15 of the largest 65,504, and those
    // that vanish, below 2^-25, are 2^-32 of the row's largest or less (of 131,072 tokens beside a
    // dominant one 2^-15 altogether; with the maximum itself as the reference it was 2^-8).
    static constexpr float kBelow = MT == KVR_DT_FP16 ? 7.0f : 0.0f;
    template <int U>
    __device__ __forceinline__ void reference(int step, int last, f32x4 (&sc)[U][RT][2], State &st) const
    {
        if ((step + U) * kStep > prefix || step + U > last) {
            const int end = min(len, last * kStep);
            // Bits first, then selects: hipcc (ROCm 7.2) loses stores of single elements of
            // the accumulators under divergent branches.
            static_for<0, U * RT>([&](auto I) {
                constexpr int u = decltype(I)::value / RT, r = decltype(I)::value % RT;
                const int t = token(step + u, 0);
                const uint32_t seen = seen4<r>(st, t, end) | seen4<r>(st, t + 16, end) << 4;
                const f32x4 x = sc[u][r][0], y = sc[u][r][1];
                auto pick = [&](int i, float z) { return seen >> i & 1 ? z : -INFINITY; };
                sc[u][r][0] = f32x4{pick(0, x[0]), pick(1, x[1]), pick(2, x[2]), pick(3, x[3])};
                sc[u][r][1] = f32x4{pick(4, y[0]), pick(5, y[1]), pick(6, y[2]), pick(7, y[3])};
            });
        }
        float top[RT];
        bool moves = false;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            top[r] = kLowest;
            static_for<0, U>([&](auto V) {
                const f32x4 x = sc[decltype(V)::value][r][0], y = sc[decltype(V)::value][r][1];
                const float z = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                      fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
                top[r] = decltype(V)::value ? fmaxf(top[r], z) : z;
            });
            top[r] *= a.scale2;
            moves = moves || top[r] > st.m[r] + (8.0f + kBelow);
        });
        if (__ballot(moves)) {
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const float t = fmaxf(row_max(top[r]) - kBelow, st.m[r]);
                const float f = __builtin_amdgcn_exp2f(st.m[r] - t);
                st.l[r] *= f;
                st.w[r] *= f;
                static_for<0, 2 * NB>([&](auto E) { st.o[r][decltype(E)::value] *= f; });
                st.m[r] = t;
            });
        }
    }

    // The weights of a row tile's scores, in the products' type: 16 bits, which the matrix
    // instructions take; 32 would be two products in place of one.  Scores, sums and outputs stay in
    // 32.  The outputs' error against 64 bits, most of it their own rounding to bfloat16, is
    // 0.0019 of them with it and 0.0017 without for one token over 1,000, 0.0018 and 0.0017 over
    // 8,192 in 8 bits, 0.0022 and 0.0017 for trees over 2,048 to 32,768 tokens.
    template <int R>
    __device__ __forceinline__ void weights(const f32x4 (&sc)[2], State &st, u32x4 (&pv)[QS]) const
    {
        constexpr int r = R;
        const f32x4 s0 = sc[0], s1 = sc[1];
        float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -st.m[r]));
        st.l[r] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pv[0][i] = pack16<MT>(x[2 * i], x[2 * i + 1]);
            if (QS == 2) {
                float y0, y1;
                unpack16<MT>(pv[0][i], y0, y1);
                pv[QS - 1][i] = pack16<MT>(x[2 * i] - y0, x[2 * i + 1] - y1);
            }
        }
    }

    // The sum of the weights as they were rounded, by a product with ones: the outputs
    // are divided by it, so that the rounding of a large weight cancels.
    __device__ __forceinline__ void count(const u32x4 (&pv)[RT][QS], State &st) const
    {
        constexpr uint32_t one = MT == KVR_DT_BF16 ? 0x3f803f80u : 0x3c003c00u;
        static_for<0, RT * QS>([&](auto I) {
            constexpr int r = decltype(I)::value / QS, p = decltype(I)::value % QS;
            st.w[r] = mfma<MT>(u32x4{one, one, one, one}, pv[r][p], st.w[r]);
        });
    }
    // O^T += V^T P^T of one value tile.
    template <int E>
    __device__ __forceinline__ void accumulate(u32x4 x, const u32x4 (&pv)[RT][QS], State &st) const
    {
        static_for<0, RT * QS>([&](auto I) {
            constexpr int r = decltype(I)::value / QS, p = decltype(I)::value % QS;
            st.o[r][E] = mfma<MT>(x, pv[r][p], st.o[r][E]);
        });
    }

    // One step from registers; returns whether values were taken out.
    __device__ __forceinline__ bool compute(int step, Stage &raw, State &st) const
    {
        f32x4 sc[1][RT][2];
        static_for<0, 2>([&](auto T) {
            constexpr int t = decltype(T)::value;
            static_for<0, RT>([&](auto R) { sc[0][decltype(R)::value][t] = f32x4{0, 0, 0, 0}; });
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value;
                scores<i, t>(key_block<i>(raw.k[t]), st, sc[0]);
            });
        });
        reference<1>(step, step + 1, sc, st);
        u32x4 pv[RT][QS];
        static_for<0, RT>([&](auto R) {
            weights<decltype(R)::value>(sc[0][decltype(R)::value], st, pv[decltype(R)::value]);
        });
        count(pv, st);
        const bool odd = clean(step, raw.v);
        static_for<0, NB>([&](auto I) {
            u32x4 x[2];
            val_tiles<decltype(I)::value>(raw.v, x);
            accumulate<2 * decltype(I)::value>(x[0], pv, st);
            accumulate<2 * decltype(I)::value + 1>(x[1], pv, st);
        });
        return odd;
    }
    template <int I, int T>
    __device__ __forceinline__ void scores(u32x4 kb, const State &st, f32x4 (&sc)[RT][2]) const
    {
        static_for<0, RT * QS>([&](auto J) {
            constexpr int r = decltype(J)::value / QS, p = decltype(J)::value % QS;
            sc[r][T] = mfma<MT>(kb, st.q[r][p][I], sc[r][T]);
        });
    }

    // A step's keys or values into LDS, converted and turned around.
    __device__ __forceinline__ void put_keys(const KR (&k)[2], uint32_t *lds) const
    {
        u32x4 *kf = reinterpret_cast<u32x4 *>(lds) + lane;
#pragma unroll
        for (int t = 0; t < 2; ++t)
            static_for<0, NB>([&](auto I) {
                kf[(t * NB + decltype(I)::value) * 64] = key_block<decltype(I)::value>(k[t]);
            });
    }
    __device__ __forceinline__ bool put_values(int step, VR &v, uint32_t *lds) const
    {
        u32x4 *vf = reinterpret_cast<u32x4 *>(lds) + 2 * NB * 64 + lane;
        const bool odd = clean(step, v);
        static_for<0, NB>([&](auto I) {
            u32x4 x[2];
            val_tiles<decltype(I)::value>(v, x);
            vf[(2 * decltype(I)::value) * 64] = x[0];
            vf[(2 * decltype(I)::value + 1) * 64] = x[1];
        });
        return odd;
    }
    __device__ __forceinline__ void clear_values(uint32_t *lds) const
    {
        u32x4 *vf = reinterpret_cast<u32x4 *>(lds) + 2 * NB * 64 + lane;
#pragma unroll
        for (int e = 0; e < 2 * NB; ++e) vf[e * 64] = u32x4{0, 0, 0, 0};
    }

    // The softmax goes before the other block's products where two row tiles a wave make both
    // long: 512 rows over 16,384 tokens 661 us against 685 on one card; with one tile 74 against 72.
    template <int P>
    __device__ __forceinline__ static void priority()
    {
        if constexpr (RT == 2) __builtin_amdgcn_s_setprio(P);
    }

    // Two steps from LDS.  Their keys, then their values, are read a group ahead of the
    // products that use them where registers allow: left to itself the compiler reads a pair of
    // fragments, waits for it and multiplies.  (Two groups ahead, or the first step's
    // outputs interleaved with the second one's weights, measured the same or slower.)
    static constexpr int G = NB == 3 ? 3 : 4;     // fragments of a group
    static constexpr int GS = 2 * NB / G;         // groups of one step's keys, or values
    static constexpr int Ahead = RT == 2 || NB == 6;   // (others: a block less on the CU)
    __device__ __forceinline__ void compute_shared(int step, int last, const uint32_t *lds,
                                                   State &st) const
    {
        const u32x4 *f = reinterpret_cast<const u32x4 *>(lds) + lane;
        u32x4 frag[Ahead + 1][G];
        auto fetch = [&](auto K) {
            constexpr int k = decltype(K)::value, u = k % (Pair * GS) / GS;
            if constexpr (k < 2 * Pair * GS) {
                static_for<0, G>([&](auto J) {
                    constexpr int j = k % GS * G + decltype(J)::value;   // within the step
                    // both tiles of keys in turn: successive products then differ in their sums
                    constexpr int at = k < Pair * GS ? j % 2 * NB + j / 2 : 2 * NB + j;
                    frag[k % (Ahead + 1)][decltype(J)::value] = f[u * (StepWords / 4) + at * 64];
                });
            }
            if constexpr (Ahead > 0)   // only vector and scalar arithmetic may pass
                __builtin_amdgcn_sched_barrier(0x406);
        };
        priority<0>();
        static_for<0, Ahead>(fetch);
        f32x4 sc[Pair][RT][2];
        static_for<0, 2 * Pair * RT>([&](auto I) {
            constexpr int i = decltype(I)::value;
            sc[i / (2 * RT)][i / 2 % RT][i % 2] = f32x4{0, 0, 0, 0};
        });
        static_for<0, Pair * GS>([&](auto K) {
            constexpr int k = decltype(K)::value;
            fetch(std::integral_constant<int, k + Ahead>{});
            static_for<0, G>([&](auto J) {
                constexpr int j = k % GS * G + decltype(J)::value;
                scores<j / 2, j % 2>(frag[k % (Ahead + 1)][decltype(J)::value], st, sc[k / GS]);
            });
        });
        priority<1>();
        reference<Pair>(step, last, sc, st);
        static_for<0, Pair>([&](auto U) {
            constexpr int u = decltype(U)::value;
            u32x4 pv[RT][QS];
            static_for<0, RT>([&](auto R) {
                weights<decltype(R)::value>(sc[u][decltype(R)::value], st, pv[decltype(R)::value]);
            });
            priority<0>();
            count(pv, st);
            static_for<0, GS>([&](auto I) {
                constexpr int k = (Pair + u) * GS + decltype(I)::value;
                fetch(std::integral_constant<int, k + Ahead>{});
                static_for<0, G>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    accumulate<decltype(I)::value * G + j>(frag[k % (Ahead + 1)][j], pv, st);
                });
            });
            priority<u == 0>();
        });
    }

    // Queries of the 16-row tiles from row r0 on; rows past the last repeat it.
    __device__ __forceinline__ void load_queries(int r0, int rows, State &st) const
    {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = min(r0 + 16 * r + (int)n, rows - 1);
            st.qi[r] = row / a.group;
            const int head = h * a.group + (row - st.qi[r] * a.group);
            st.word[r] = a.mask && a.words == 1 ? a.mask[q0 + st.qi[r]] : 0;
            const char *src = a.q.p + ((int64_t)(q0 + st.qi[r]) * a.q.token_stride +
                                       (int64_t)head * a.q.head_stride) * 2;
            const uint32_t flip = a.negate ? 0x80008000u : 0u;
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value, s = KR::slab_of(i), start = KR::start(s);
                const int d = start * 32 + g * KR::width(s) * 8 + (i - start) * 8;
                u32x4 x = *reinterpret_cast<const u32x4 *>(src + d * 2) ^ flip;
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
                    st.q[r][QS - 1][i] = lo;
                }
                st.q[r][0][i] = x;
            });
            st.m[r] = kLowest;
            st.l[r] = 0.0f;
            st.w[r] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 2 * NB; ++e) st.o[r][e] = f32x4{0, 0, 0, 0};
        }
    }

    // W adjacent elements (2, 4 or 8) of a row of the output, or of a part's.
    template <int W>
    __device__ __forceinline__ void store(const Part &p, int64_t cell, int r0, int row, int d,
                                          const float *x, float top, float sum, float norm) const
    {
        if (p.parts != 1) {
            float *y = a.part_o + (cell * BlockRows + row) * D + d;
#pragma unroll
            for (int e = 0; e < W; ++e) y[e] = x[e];
            if (d == 0) a.part_ml[cell * BlockRows + row] = float4{top, sum, norm, 0.0f};
            return;
        }
        const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
        const int i0 = (r0 + row) / a.group;
        const int head = h * a.group + (r0 + row - i0 * a.group);
        uint32_t *y = reinterpret_cast<uint32_t *>(
            a.out.p + ((int64_t)(q0 + i0) * a.out.token_stride + (int64_t)head * a.out.head_stride + d) * 2);
        uint32_t w[W / 2];
#pragma unroll
        for (int e = 0; e < W / 2; ++e) w[e] = pack16<QT>(x[2 * e] * inv, x[2 * e + 1] * inv);
        if constexpr (W == 8) *reinterpret_cast<u32x4 *>(y) = u32x4{w[0], w[1], w[2], w[3]};
        else if constexpr (W == 4) *reinterpret_cast<u32x2 *>(y) = u32x2{w[0], w[1]};
        else *y = w[0];
        if (d == 0 && a.lse)
            a.lse[(int64_t)(q0 + i0) * a.q_heads + head] =
                sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }

    __device__ __forceinline__ void run(uint32_t *lds)
    {
        // Heads fastest: with eight or a multiple of them the row blocks of one part, which
        // follow each other, land on one XCD (block number mod 8) and share its L2.
        const int item = blockIdx.x / a.c.n_heads;
        h = blockIdx.x - item * a.c.n_heads;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        Pages where[PF];
        auto table_row = [&](int b) { pages = a.pages + (int64_t)b * a.pages_stride; };
        auto first_pages = [&](int step) {
#pragma unroll
            for (int i = 0; i < PF; ++i) where[i] = look_up(step + wave + i * Waves);
        };
        // Beside the lengths (in the shared kernel the same made the loop 5 % slower).
        if (!Shared && a.direct) {
            table_row(item / a.direct);
            first_pages(0);
        }
        const Part p = find_part(a, item);
        if (p.b < 0) return;
        const int rows = p.nq * a.group, r0 = p.rb * BlockRows;
        len = p.len;
        prefix = p.len - p.nq;
        q0 = p.q0;
        if (Shared || !a.direct) table_row(p.b);
        if (!Shared && !a.direct) first_pages(p.first);
        if constexpr (Shared) run_shared(p, wave, r0, rows, lds);
        else run_split(p, wave, r0, rows, where, reinterpret_cast<float *>(lds));
    }

    // Few rows: every wave has all of the block's rows and every n-th step.
    __device__ __forceinline__ void run_split(const Part &p, int wave, int r0, int rows,
                                              Pages (&where)[PF], float *lds)
    {
        State st;
        Stage raw[PF];
        bool odd = false;
        int s = p.first + wave;
#pragma unroll
        for (int i = 0; i < PF; ++i)
            if (s + i * Waves < p.last) {
                load(s + i * Waves, where[i], raw[i]);
                where[i] = look_up(s + (PF + i) * Waves);
            }
        load_queries(r0, rows, st);
        for (; s < p.last; s += PF * Waves) {
#pragma unroll
            for (int i = 0; i < PF; ++i) {
                const int at = s + i * Waves;
                if (at < p.last) {
                    odd |= compute(at, raw[i], st);
                    if (at + PF * Waves < p.last) {
                        load(at + PF * Waves, where[i], raw[i]);
                        where[i] = look_up(at + 2 * PF * Waves);
                    }
                }
            }
        }
        // join the waves: maxima first, then sums and values in wave order
        float *sm = lds, *sl = sm + Waves * BlockRows, *sw = sl + Waves * BlockRows,
              *so = sw + Waves * BlockRows;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            st.l[r] = row_sum(st.l[r]);
            if (g == 0) {
                sm[wave * BlockRows + 16 * r + n] = st.m[r];
                sl[wave * BlockRows + 16 * r + n] = st.l[r];
                sw[wave * BlockRows + 16 * r + n] = st.w[r][0];
            }
        }
        odd = __syncthreads_or(odd);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = kLowest;
#pragma unroll
            for (int w = 0; w < Waves; ++w) top = fmaxf(top, sm[w * BlockRows + 16 * r + n]);
            const float f = __builtin_amdgcn_exp2f(st.m[r] - top);
#pragma unroll
            for (int e = 0; e < 2 * NB; ++e) st.o[r][e] *= f;
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float *row = so + (wave * BlockRows + 16 * r + n) * LdsRow;
            static_for<0, 2 * NB>([&](auto E) {
                // tile e of its slab: element (4 g + i) * W + e - e0 of the slab
                constexpr int e = decltype(E)::value, slab = VR::slab_of(e);
                constexpr int e0 = VR::first(slab), W = VR::width(slab);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    row[16 * e0 + (4 * g + i) * W + (e - e0)] = st.o[r][e][i];
            });
        }
        __syncthreads();
        // rows out: eight elements a thread
        const int64_t cell = blockIdx.x;
        for (int i = threadIdx.x; i < BlockRows * (D / 8); i += 64 * Waves) {
            const int row = i / (D / 8), d = 8 * (i - row * (D / 8));
            if (r0 + row >= rows) break;
            float top = kLowest, sum = 0.0f, norm = 0.0f;
#pragma unroll
            for (int w = 0; w < Waves; ++w) top = fmaxf(top, sm[w * BlockRows + row]);
#pragma unroll
            for (int w = 0; w < Waves; ++w) {
                const float f = __builtin_amdgcn_exp2f(sm[w * BlockRows + row] - top);
                sum += sl[w * BlockRows + row] * f;
                norm += sw[w * BlockRows + row] * f;
            }
            float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < Waves; ++w) {
                const float *y = so + (w * BlockRows + row) * LdsRow + d;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += y[e];
            }
            if (odd) add_odd<8>(p, r0 + row, d, x);
            store<8>(p, cell, r0, row, d, x, top, sum, norm);
        }
    }

    // The loop of a wave that brings the keys (or the values) of step `mine` of every
    // tile into LDS.  Two copies of it, so that the keys and the values in flight take
    // the same registers.
    template <bool Keys>
    __device__ __forceinline__ bool walk(const Part &p, int mine, bool active, uint32_t *lds,
                                         State &st) const
    {
        std::conditional_t<Keys, Stage, VR> raw;   // of Stage only the keys
        bool odd = false;
        Pages where = look_up(p.first + mine);
        auto fetch = [&](int s) {
            if (s + mine >= p.last) return;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const Where at = locate(s + mine, t, where);
                if constexpr (Keys) load_keys(at, raw.k[t]);
                else load_values(at, t, raw);
            }
            where = look_up(s + Tile + mine);
        };
        fetch(p.first);
        for (int s = p.first; s < p.last; s += Tile) {
            uint32_t *to = lds + mine * StepWords;
            if (s + mine < p.last) {
                if constexpr (Keys) put_keys(raw.k, to);
                else odd = put_values(s + mine, raw, to) || odd;
            } else if (!Keys) {
                clear_values(to);   // beyond the part: weights of zero meet zeros
            }
            fetch(s + Tile);
            __syncthreads();
            if (active)
                for (int u = 0; u < Tile && s + u < p.last; u += Pair)
                    compute_shared(s + u, p.last, lds + u * StepWords, st);
            __syncthreads();
        }
        return odd;
    }

    // Many rows: the waves divide the block's rows and all work on every step; half of
    // them bring keys into LDS and half values.
    __device__ __forceinline__ void run_shared(const Part &p, int wave, int r0, int rows, uint32_t *lds)
    {
        const int w0 = 16 * RT * wave;
        const bool active = r0 + w0 < rows;
        State st;
        load_queries(r0 + w0, rows, st);
        bool odd = wave < Tile ? walk<true>(p, wave, active, lds, st)
                               : walk<false>(p, wave - Tile, active, lds, st);
        odd = __syncthreads_or(odd);
        const int64_t cell = blockIdx.x;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const int row = w0 + 16 * r + (int)n;
            const float sum = row_sum(st.l[r]);
            if (r0 + row >= rows) return;
            static_for<0, VR::slabs>([&](auto S) {
                constexpr int e0 = VR::first(decltype(S)::value), W = VR::width(decltype(S)::value);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x[W];
#pragma unroll
                    for (int e = 0; e < W; ++e) x[e] = st.o[r][e0 + e][i];
                    const int d = 16 * e0 + (4 * (int)g + i) * W;
                    if (odd) add_odd<W>(p, r0 + row, d, x);
                    store<W>(p, cell, r0, row, d, x, st.m[r], sum, st.w[r][0]);
                }
            });
        });
    }
};

template <int FMT, int QT, int NB, int RT, int PF, bool Shared, int Waves>
__global__ __launch_bounds__(64 * Waves, 2) void attention_kernel(Attention a)
{
    using K = Kernel<FMT, QT, NB, RT, PF, Shared, Waves>;
    __shared__ __align__(16) uint32_t lds[K::LdsWords];
    K k(a);
    k.run(lds);
}

// The kernel that the plan names: its workspace and grid hold this one's blocks only.
template <int FMT, int QT, int NB, int RT, int PF, bool Shared, int Waves>
hipError_t launch_kernel(const Attention &a, dim3 grid, hipStream_t stream)
{
    if (a.block_rows != Kernel<FMT, QT, NB, RT, PF, Shared, Waves>::BlockRows || a.waves != Waves)
        return hipErrorInvalidValue;
    attention_kernel<FMT, QT, NB, RT, PF, Shared, Waves><<<grid, 64 * Waves, 0, stream>>>(a);
    return hipGetLastError();
}

// One launch for a format, query type and head size, by the plan.
template <int FMT, int QT, int NB, int RT, int Waves>
hipError_t launch_split(const Attention &a, dim3 grid, hipStream_t stream)
{
    // steps in flight: what the registers left by queries and accumulators hold
    constexpr int stage = NB * Fmt<FMT>::B8;   // registers of one step's keys and values
    constexpr bool quant = Fmt<FMT>::Quant, two = quant && QT == KVR_DT_FP16;
    constexpr int room = (RT == 2 ? (quant ? 32 : 64) : quant ? 64 : 128) / stage;
    constexpr int PF = room < 1 || NB * (two ? 2 : 1) > 8 || NB == 8 ? 1 : room > 3 ? 3 : room;
    return launch_kernel<FMT, QT, NB, RT, PF, false, Waves>(a, grid, stream);
}

template <int FMT, int QT, int NB>
hipError_t launch_nb(const Attention &a, dim3 grid, hipStream_t stream)
{
    if constexpr (NB <= 4) {   // heads beyond 128 take one row tile a wave
        if (a.row_tiles == 2 && a.shared)
            return launch_kernel<FMT, QT, NB, 2, 1, true, 4>(a, grid, stream);
        if (a.row_tiles == 2) return launch_split<FMT, QT, NB, 2, 4>(a, grid, stream);
    }
    if (a.shared) return launch_kernel<FMT, QT, NB, 1, 1, true, 4>(a, grid, stream);
    return a.waves == 8 ? launch_split<FMT, QT, NB, 1, 8>(a, grid, stream)
                        : launch_split<FMT, QT, NB, 1, 4>(a, grid, stream);
}

template <int FMT, int QT>
hipError_t launch_dim(const Attention &a, dim3 grid, hipStream_t stream)
{
    switch (a.c.dim) {
    case 64: return launch_nb<FMT, QT, 2>(a, grid, stream);
    case 96: return launch_nb<FMT, QT, 3>(a, grid, stream);
    case 192: return launch_nb<FMT, QT, 6>(a, grid, stream);
    case 256: return launch_nb<FMT, QT, 8>(a, grid, stream);
    default: return launch_nb<FMT, QT, 4>(a, grid, stream);
    }
}

}  // namespace
}  // namespace kv
}  // namespace kvr
