// Attention of prompts whose keys have a part of each head's own and a rotated part that
// all heads share:
//   s_ij = scale (q_i[: nope] . k_j + q_i[nope :] . r_j),  out_i = sum_j softmax_j(s_ij) v_j,
// one pass over the keys with the running maximum and sum.  Matrix instructions bound it: 2 (2
// nope + rot) operations a query, head and key that it sees.
//
// They compute S^T = K Q^T and O^T = V^T P^T (16x16x32), so that a lane owns one query (lane mod
// 16) and P^T leaves the first product in the layout that the second one takes.  A block has
// four waves of 32 queries of one head; 64 keys and values (a step) go from memory to LDS
// without passing through registers, while the step before is worked on, 16-byte chunks
// exchanged within a row so that reading along it (keys) and across it (values, ds_read_b64_tr_b16)
// spreads over the banks.  A causal block ends at the last key that its queries see, a wave at its
// own; blocks with the most keys come first.  Where the blocks are fewer than the GPU holds, the
// keys of each are cut into parts, which join_kernel joins.  Scores, sums and outputs are held in 32
// bits; weights are rounded to the inputs' type and the outputs divided by the sum of the rounded ones.
//
// One prompt of 8,192 tokens, 32 heads of 128 + 64: 690 us a call in a steady run (670 to 750 by card), 996
// TFLOP/s, where a large product reaches 1,135; the first dozen calls after a pause take 770 to 950.  Two chunks of 509 after 16,384 tokens: 268 us, 12 of them the joining.
// Fragments read in groups ahead of the products, as attention over latents does, spilled
// registers: 967 against 805 us on the same card.
#include <algorithm>

#include "kvr_latent_attention.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kKeys = 64;   // of a step
constexpr int kBlockRows = 128;   // queries of a block

// LDS position of chunk c (16 bytes) of row r, rows of C chunks.
template <int C>
__device__ __forceinline__ int swizzle(int r)
{
    return C >= 16 ? r & 15 : C == 8 ? r >> 1 & 7 : r >> 2 & 3;
}

struct Item {   // what a block works on
    int b;            // sequence; -1: nothing to do
    int rb;           // block of its queries
    int nq, q0, nk, k0;
};

__device__ __forceinline__ bool prompt_sequence(const Prompt &p, int b, int &nq, int &q0, int &nk, int &k0)
{
    q0 = p.cu_q[b];
    nq = p.cu_q[b + 1] - q0;
    k0 = p.cu_k[b];
    nk = p.cu_k[b + 1] - k0;
    const bool ok = q0 >= 0 && nq >= 0 && nq <= p.max_q && (int64_t)q0 + nq <= p.n_queries &&
                    k0 >= 0 && nk >= 0 && nk <= p.max_k && (int64_t)k0 + nk <= p.n_keys;
    if (!ok) {
        if (p.status) *p.status = KVR_E_DOMAIN;
        nq = nk = 0;
    }
    return ok;
}

// Blocks of sequences in order, the last queries of each first.
__device__ __forceinline__ Item find_item(const Prompt &p, int item)
{
    int base = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += 64) {
        const int b = b0 + (threadIdx.x & 63);
        int nq = 0, q0 = 0, nk = 0, k0 = 0;
        if (b < p.n_seqs) prompt_sequence(p, b, nq, q0, nk, k0);
        const int blocks = (nq + p.block_rows - 1) / p.block_rows;
        const int upto = wave_incl_scan(blocks);
        const uint64_t hit = __ballot(base + upto > item);
        if (hit) {
            const int w = __ffsll((unsigned long long)hit) - 1;
            Item x;
            x.b = b0 + w;
            x.rb = base + lane_value(upto, w) - 1 - item;
            x.nq = lane_value(nq, w), x.q0 = lane_value(q0, w);
            x.nk = lane_value(nk, w), x.k0 = lane_value(k0, w);
            return x;
        }
        base += lane_value(upto, 63);
    }
    Item none{};
    none.b = -1;
    return none;
}

template <int MT, int NOPE, int ROT>
struct PromptKernel {
    static constexpr int KB = NOPE / 32, SB = ROT / 32, NB = KB + SB;   // blocks of 32 elements
    static constexpr int VT = NOPE / 16;                                // value tiles
    static constexpr int BlockRows = kBlockRows, WaveRows = BlockRows / 4, RT = WaveRows / 16;
    // LDS bytes of a step: own keys, shared keys, values
    static constexpr int OwnBytes = kKeys * NOPE * 2, SharedBytes = kKeys * ROT * 2;
    static constexpr int Tile = 2 * OwnBytes + SharedBytes, ValuesAt = OwnBytes + SharedBytes;
    static constexpr int LdsBytes = 2 * Tile;

    struct State {
        u32x4 q[RT][NB];
        f32x4 o[RT][VT];
        float m[RT], l[RT], w[RT];   // reference (log2); this lane's part of the sum of the weights, and as rounded
        int last[RT];    // the last key that the lane's query sees (-1: none)
    };

    const Prompt &p;
    const int n, g, lane, wave;
    int h, kvh, nk, k0, q0, nq;
    uint32_t own_at[NOPE == 128 ? 4 : 2], shared_at[SB], val_at[NOPE == 128 ? 8 : 4];

    __device__ PromptKernel(const Prompt &a)
        : p(a), n(threadIdx.x & 15), g((threadIdx.x & 63) >> 4), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6))
    {
#pragma unroll
        for (int i = 0; i < KB; ++i)
            own_at[i] = n * (NOPE * 2) + (((4 * i + g) ^ swizzle<NOPE / 8>(n)) << 4);
#pragma unroll
        for (int i = 0; i < SB; ++i)
            shared_at[i] = OwnBytes + n * (ROT * 2) + (((4 * i + g) ^ swizzle<ROT / 8>(n)) << 4);
        const int r = 4 * g + (n >> 2);
#pragma unroll
        for (int e = 0; e < VT; ++e)
            val_at[e] = ValuesAt + r * (NOPE * 2) +
                        (((2 * e + ((n & 3) >> 1)) ^ swizzle<NOPE / 8>(r)) << 4) + ((n & 1) << 3);
    }

    // Rows of C chunks of a step into LDS; rows past the sequence's last key read as that one.
    template <int C, bool Whole>
    __device__ __forceinline__ void bring(const Rows &from, int64_t head, int first, uint32_t to) const
    {
        constexpr int Loads = kKeys * C / 64, PerLoad = 64 / C;   // rows of a load
        const int64_t stride = from.token_stride * 2;
        const char *base = from.p + uniform((int64_t)(k0 + first) * stride + head * from.head_stride * 2);
#pragma unroll
        for (int j0 = 0; j0 < Loads; j0 += 4) {
            const int j = j0 + wave, r = j * PerLoad + lane / C;
            const uint32_t c = 16 * ((lane & (C - 1)) ^ swizzle<C>(r));
            if (Whole)
                load_to_lds(base + j * PerLoad * stride, lane / C * (uint32_t)stride + c, to + j * 1024);
            else load_to_lds(base + min(r, nk - 1 - first) * stride + c, to + j * 1024);
        }
    }
    template <bool Whole>
    __device__ __forceinline__ void bring_step(int first, uint32_t tile) const
    {
        bring<NOPE / 8, Whole>(p.k, kvh, first, tile);
        bring<ROT / 8, Whole>(p.shared, 0, first, tile + OwnBytes);
        bring<NOPE / 8, Whole>(p.v, kvh, first, tile + ValuesAt);
    }
    __device__ __forceinline__ void fetch(int step, uint32_t tile) const
    {
        if ((step + 1) * kKeys <= nk) bring_step<true>(step * kKeys, tile);
        else bring_step<false>(step * kKeys, tile);
    }

    static constexpr float kBelow = MT == KVR_DT_FP16 ? 7.0f : 0.0f;

    // sure: every query of the wave sees every key of the step.
    __device__ __forceinline__ bool compute(int step, bool sure, const char *tile, State &st) const
    {
        bool odd = false;
        if (!sure) {   // a weight of zero would not hide an infinity or a NaN
            u16x2 most = {0, 0};
#pragma unroll 4
            for (int i = 0; i < OwnBytes / 1024; ++i) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(tile + ValuesAt + i * 1024 + lane * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) keep_most<MT>(x[k], most);
            }
            odd = any_odd<MT>(most);
        }
        f32x4 sc[RT][4];
        u32x4 pv[RT][2];
        static_for<0, 4 * RT>([&](auto I) {
            sc[decltype(I)::value / 4][decltype(I)::value % 4] = f32x4{0, 0, 0, 0};
        });
        static_for<0, 4>([&](auto T) {
            constexpr int t = decltype(T)::value;
            static_for<0, NB>([&](auto I) {
                constexpr int i = decltype(I)::value;
                const char *at = tile + (i < KB ? own_at[i < KB ? i : 0] + t * 16 * NOPE * 2
                                                : shared_at[i < KB ? 0 : i - KB] + t * 16 * ROT * 2);
                const u32x4 x = *reinterpret_cast<const u32x4 *>(at);
                static_for<0, RT>([&](auto R) {
                    constexpr int r = decltype(R)::value;
                    sc[r][t] = mfma<MT>(x, st.q[r][i], sc[r][t]);
                });
            });
        });
        if (!sure) {
            static_for<0, 4 * RT>([&](auto I) {
                constexpr int r = decltype(I)::value / 4, t = decltype(I)::value % 4;
                const int left = st.last[r] - (step * kKeys + 16 * t + 4 * g);   // < 0: none of the four
                const f32x4 x = sc[r][t];
                sc[r][t] = f32x4{left >= 0 ? x[0] : -INFINITY, left >= 1 ? x[1] : -INFINITY,
                                 left >= 2 ? x[2] : -INFINITY, left >= 3 ? x[3] : -INFINITY};
            });
        }
        float top[RT];
        bool moves = false;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            float z[4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
                z[t] = fmaxf(fmaxf(sc[r][t][0], sc[r][t][1]), fmaxf(sc[r][t][2], sc[r][t][3]));
            top[r] = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) * p.scale2;
            moves = moves || top[r] > st.m[r] + (8.0f + kBelow);
        });
        if (__ballot(moves)) {
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                const float t = fmaxf(row_max(top[r]) - kBelow, st.m[r]);
                const float f = __builtin_amdgcn_exp2f(st.m[r] - t);
                st.l[r] *= f;
                st.w[r] *= f;
                static_for<0, VT>([&](auto E) { st.o[r][decltype(E)::value] *= f; });
                st.m[r] = t;
            });
        }
        static_for<0, 2 * RT>([&](auto I) {
            constexpr int r = decltype(I)::value / 2, u = decltype(I)::value % 2;
            const f32x4 s0 = sc[r][2 * u], s1 = sc[r][2 * u + 1];
            float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], p.scale2, -st.m[r]));
            st.l[r] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pv[r][u][i] = pack16<MT>(x[2 * i], x[2 * i + 1]);
                st.w[r] = add_pair<MT>(pv[r][u][i], st.w[r]);   // what the outputs are divided by
            }
        });
        static_for<0, 2 * VT>([&](auto E) {
            constexpr int u = decltype(E)::value / VT, e = decltype(E)::value % VT;
            const char *at = tile + val_at[e] + u * 32 * NOPE * 2;
            const u32x2 lo = read_across(at), hi = read_across(at + 16 * NOPE * 2);
            uint32_t w[4] = {lo[0], lo[1], hi[0], hi[1]};
            if (odd) {   // (in registers: another wave may see all these keys)
#pragma unroll
                for (int i = 0; i < 4; ++i) clear_odd2<MT>(w[i]);
            }
            const u32x4 x = {w[0], w[1], w[2], w[3]};
            static_for<0, RT>([&](auto R) {
                constexpr int r = decltype(R)::value;
                st.o[r][e] = mfma<MT>(x, pv[r][u], st.o[r][e]);
            });
        });
        return odd;
    }

    // The infinities and NaN that compute() took out, among keys from `from` on that the query sees.
    __device__ __forceinline__ void add_odd(int from, int upto, int d, float *x) const
    {
        constexpr uint32_t e = MT == KVR_DT_FP16 ? 0x7c00u : 0x7f80u;
        for (int t = from; t <= upto; ++t) {
            const uint16_t *row = reinterpret_cast<const uint16_t *>(p.v.p) +
                                  (int64_t)(k0 + t) * p.v.token_stride + (int64_t)kvh * p.v.head_stride + d;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((row[i] & e) == e) {
                    float y, z;
                    unpack16<MT>(row[i], y, z);
                    x[i] += y;
                }
        }
    }

    __device__ __forceinline__ void run(char *lds)
    {
        // heads fastest: with a multiple of eight of them, a head's blocks are on one XCD
        const int per = p.q_heads;
        const int at = block_of_grid() / per, part = at / p.max_items, item = at - part * p.max_items;
        h = block_of_grid() - at * per;
        if (part >= p.parts) return;   // beyond the last block
        const Item x = find_item(p, item);
        if (x.b < 0) return;
        kvh = h / p.group;
        nk = uniform(x.nk), k0 = uniform(x.k0), q0 = uniform(x.q0), nq = uniform(x.nq);
        const int r0 = x.rb * BlockRows, w0 = r0 + WaveRows * wave;
        const int past = nk - nq;   // query i sees the keys up to past + i
        State st;
        const uint32_t flip = p.negate ? 0x80008000u : 0u;
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const int i = min(w0 + 16 * r + n, nq - 1);
            st.last[r] = p.causal ? past + i : nk - 1;
            const char *src = p.q.p + ((int64_t)(q0 + i) * p.q.token_stride + (int64_t)h * p.q.head_stride) * 2;
            static_for<0, NB>([&](auto I) {
                constexpr int b = decltype(I)::value;
                st.q[r][b] = *reinterpret_cast<const u32x4 *>(src + (b * 32 + g * 8) * 2) ^ flip;
            });
            st.m[r] = kLowest;
            st.l[r] = 0.0f;
            st.w[r] = 0.0f;
            static_for<0, VT>([&](auto E) { st.o[r][decltype(E)::value] = f32x4{0, 0, 0, 0}; });
        });
        // steps of the block, and of its part; the wave's keys [0, see), all of it to `all`
        auto seen = [&](int i) { return p.causal ? max(0, past + min(i, nq - 1) + 1) : nk; };
        const int steps = (seen(r0 + BlockRows - 1) + kKeys - 1) / kKeys;
        const int first = (int)((int64_t)steps * part / p.parts);
        const int end = (int)((int64_t)steps * (part + 1) / p.parts);
        const int see = w0 < nq ? seen(w0 + WaveRows - 1) : 0, all = w0 < nq ? seen(w0) : 0;
        bool odd = false;
        const uint32_t lds_at = lds_address(lds);
        if (first < end) fetch(first, lds_at);
        for (int s = first; s < end; ++s) {
            wait_loads<0>();
            block_barrier();   // the step's rows are there, the other buffer has been read
            if (s + 1 < end) fetch(s + 1, lds_at + ((s + 1 - first) & 1) * Tile);
            if (s * kKeys < see)
                odd |= compute(s, (s + 1) * kKeys <= all, lds + ((s - first) & 1) * Tile, st);
        }
        __syncthreads();
        odd = block_any(odd, reinterpret_cast<uint32_t *>(lds));
        static_for<0, RT>([&](auto R) {
            constexpr int r = decltype(R)::value;
            const int i = w0 + 16 * r + n;
            const float sum = row_sum(st.l[r]), norm = row_sum(st.w[r]);
            if (i >= nq) return;
            const int64_t cell = ((int64_t)at * p.q_heads + h) * BlockRows + (i - r0);
            static_for<0, VT>([&](auto E) {
                constexpr int e = decltype(E)::value;
                float y[4] = {st.o[r][e][0], st.o[r][e][1], st.o[r][e][2], st.o[r][e][3]};
                const int d = 16 * e + 4 * g;
                if (odd) add_odd(max(first, all / kKeys) * kKeys, min(st.last[r], end * kKeys - 1), d, y);
                if (p.parts > 1) {
                    *reinterpret_cast<f32x4 *>(p.part_o + cell * NOPE + d) = f32x4{y[0], y[1], y[2], y[3]};
                } else {
                    const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
                    char *to = p.out.p + ((int64_t)(q0 + i) * p.out.token_stride + (int64_t)h * p.out.head_stride + d) * 2;
                    *reinterpret_cast<u32x2 *>(to) = u32x2{pack16<MT>(y[0] * inv, y[1] * inv),
                                                           pack16<MT>(y[2] * inv, y[3] * inv)};
                }
            });
            if (g == 0) {
                if (p.parts > 1)
                    p.part_ml[cell] = float4{st.m[r], sum, norm, 0.0f};
                else if (p.lse)
                    p.lse[(int64_t)(q0 + i) * p.q_heads + h] =
                        sum == 0.0f ? -INFINITY : (st.m[r] + __builtin_amdgcn_logf(sum)) * kLn2;
            }
        });
    }
};

template <int MT, int NOPE, int ROT>
__global__ __launch_bounds__(256, 2) void prompt_kernel(Prompt p)
{
    using K = PromptKernel<MT, NOPE, ROT>;
    __shared__ __align__(1024) char lds[K::LdsBytes];
    K k(p);
    k.run(lds);
}

// Joins the parts of 8 or 16 queries of a block: NOPE / 4 lanes each, in the order of the parts.  Memory
// bounds it: 32 MB in 11.5 us.
template <int MT, int NOPE>
__global__ __launch_bounds__(256) void join_kernel(Prompt p)
{
    constexpr int Lanes = NOPE / 4, Rows = 256 / Lanes;
    const int per = p.block_rows / Rows;   // blocks of each block of queries
    const int at = block_of_grid() / per, piece = block_of_grid() - at * per;
    const int item = at / p.q_heads, h = at - item * p.q_heads;
    if (item >= p.max_items) return;   // beyond the last block
    const Item x = find_item(p, item);
    if (x.b < 0) return;
    const int row = piece * Rows + threadIdx.x / Lanes, d = 4 * (threadIdx.x & (Lanes - 1));
    const int r0 = x.rb * p.block_rows;
    if (r0 + row >= x.nq) return;
    const int64_t next = (int64_t)p.max_items * p.q_heads * p.block_rows;   // cells from part to part
    const int64_t cell = ((int64_t)item * p.q_heads + h) * p.block_rows + row;
    float top = kLowest;
    for (int k = 0; k < p.parts; ++k) top = fmaxf(top, p.part_ml[cell + k * next].x);
    f32x4 acc = {0, 0, 0, 0};
    float sum = 0.0f, norm = 0.0f;
#pragma unroll 4
    for (int k = 0; k < p.parts; ++k) {
        const float4 ml = p.part_ml[cell + k * next];
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        sum += f * ml.y;
        norm += f * ml.z;
        acc += f * *reinterpret_cast<const f32x4 *>(p.part_o + (cell + k * next) * NOPE + d);
    }
    const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
    const int64_t q = x.q0 + r0 + row;
    char *to = p.out.p + (q * p.out.token_stride + (int64_t)h * p.out.head_stride + d) * 2;
    *reinterpret_cast<u32x2 *>(to) = u32x2{pack16<MT>(acc[0] * inv, acc[1] * inv),
                                           pack16<MT>(acc[2] * inv, acc[3] * inv)};
    if (d == 0 && p.lse)
        p.lse[q * p.q_heads + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int MT, int NOPE, int ROT>
hipError_t launch_rows(const Prompt &p, hipStream_t stream)
{
    const int64_t blocks = (int64_t)p.max_items * p.q_heads;
    prompt_kernel<MT, NOPE, ROT><<<grid_of(blocks * p.parts), 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    join_kernel<MT, NOPE><<<grid_of(blocks * (p.block_rows / (1024 / NOPE))), 256, 0, stream>>>(p);
    return hipGetLastError();
}

template <int MT, int NOPE>
hipError_t launch_rot(const Prompt &p, hipStream_t stream)
{
    return p.rot == 64 ? launch_rows<MT, NOPE, 64>(p, stream) : launch_rows<MT, NOPE, 32>(p, stream);
}

template <int MT>
hipError_t launch_nope(const Prompt &p, hipStream_t stream)
{
    return p.nope == 128 ? launch_rot<MT, 128>(p, stream) : launch_rot<MT, 64>(p, stream);
}

constexpr int kSlots = 512;   // blocks that are resident at once

}  // namespace

size_t plan_prompt(Prompt &p)
{
    p.block_rows = kBlockRows;
    // (with all heads at most 2^36 / 128 + 2^24)
    p.max_items = (int32_t)std::max<int64_t>(
        1, std::min<int64_t>((int64_t)p.n_seqs * cdiv(p.max_q, p.block_rows),
                             p.n_queries / p.block_rows + p.n_seqs));
    const int64_t blocks = (int64_t)p.max_items * p.q_heads;
    const int64_t steps = cdiv(p.max_k, kKeys);
    // Parts of eight steps or more (us a call, joining included, against four or more: one head of 500 tokens
    // 22 and 18, of 900 32 and 21, of 1,500 26 and 21, of 4,000 33 and 35; eight heads of 900 33 and 25, of
    // 1,500 33 and 35; 32 heads of 500 22 and 26, of 900 34 and 42; two chunks of 509 behind a long past
    // alike): eight favours many heads, four would favour the few.
    p.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kSlots / blocks, steps / 8));
    if (p.parts == 1) return 0;
    return (size_t)p.parts * blocks * p.block_rows * (p.nope + 4) * sizeof(float);
}

hipError_t launch_prompt(const Prompt &p, hipStream_t stream)
{
    return p.q.dtype == KVR_DT_FP16 ? launch_nope<KVR_DT_FP16>(p, stream) : launch_nope<KVR_DT_BF16>(p, stream);
}

}  // namespace kv
}  // namespace kvr
