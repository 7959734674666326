// Attention over the paged cache: the launch plan, and the kernel that joins the
// parts of sequences that were cut.
#include <algorithm>

#include "kvr_parts.h"

namespace kvr {
namespace kv {
namespace {

// Joins the parts of one row: dim / 4 lanes x groups of parts, each group over its
// share of the parts, then the groups in order.
template <int QT>
__global__ __launch_bounds__(256) void combine_kernel(Attention a, int dim)
{
    __shared__ float so[1024];   // [groups][dim]
    __shared__ float sl[32];
    const int nh = a.c.n_heads;
    const int rows16 = 16 * a.row_tiles;
    // block: (query row slot, head, sequence)
    const int row = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    int len, nq, q0;
    sequence(a, b, len, nq, q0);
    if (row >= nq * a.group) return;
    // this sequence's parts
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int le = 0, nn = 0, qq;
        if (b0 + lane < a.n_seqs) sequence(a, b0 + lane, le, nn, qq);
        total += wave_sum(steps_of(le, nn));
    }
    const int per = part_steps(a, total);
    const int parts = (steps_of(len, nq) + per - 1) / per;
    if (parts <= 1) return;
    int base = 0;
    for (int b0 = 0; b0 < b; b0 += 64) {
        int le = 0, nn = 0, qq;
        if (b0 + lane < b) sequence(a, b0 + lane, le, nn, qq);
        base += wave_sum((steps_of(le, nn) + per - 1) / per);
    }
    const int rb = row / rows16, rr = row - rb * rows16;
    auto cell = [&](int p) {
        return (((int64_t)(base + p) * nh + h) * a.row_blocks + rb) * rows16 + rr;
    };
    float top = kLowest;
    for (int p = lane; p < parts; p += 64) top = fmaxf(top, a.part_ml[2 * cell(p)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const int cols = dim / 4;                 // 8 to 64 lanes of four elements
    const int groups = 256 / cols;
    const int grp = threadIdx.x / cols, c = threadIdx.x - grp * cols;
    f32x4 acc = {0, 0, 0, 0};
    float sum = 0.0f;
    if (grp < groups) {
#pragma unroll 4
        for (int p = grp; p < parts; p += groups) {
            const int64_t at = cell(p);
            const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * at] - top);
            sum += f * a.part_ml[2 * at + 1];
            acc += f * *reinterpret_cast<const f32x4 *>(a.part_o + at * dim + 4 * c);
        }
        *reinterpret_cast<f32x4 *>(so + grp * dim + 4 * c) = acc;
        if (c == 0) sl[grp] = sum;
    }
    __syncthreads();
    const int tid = threadIdx.x;
    if (tid < dim / 8) {
        float x[8] = {};
        float s = 0.0f;
        for (int p = 0; p < groups; ++p) {
            s += sl[p];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += so[p * dim + 8 * tid + e];
        }
        const float inv = s == 0.0f ? 0.0f : 1.0f / s;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= inv;
        const int i0 = row / a.group;
        const int head = h * a.group + (row - i0 * a.group);
        store8<QT>(a.out.p + ((int64_t)(q0 + i0) * a.out.token_stride +
                              (int64_t)head * a.out.head_stride + 8 * tid) * 2, x);
        if (tid == 0 && a.lse)
            a.lse[(int64_t)(q0 + i0) * a.q_heads + head] =
                s == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(s)) * kLn2;
    }
}

constexpr int kSlots = 1024;   // blocks that the parts are planned for

}  // namespace

size_t plan_attention(Attention &a)
{
    const int64_t rows = (int64_t)a.max_q * a.group;
    a.row_tiles = rows <= 16 ? 1 : 2;
    a.row_blocks = (int32_t)cdiv(rows, 16 * a.row_tiles);
    a.target = (int32_t)std::max<int64_t>(1, kSlots / ((int64_t)a.c.n_heads * a.row_blocks));
    a.min_steps = 4 * kWaves;
    const int64_t longest = cdiv(a.max_kv, kStep);
    // ceil per sequence of at least min_steps, and about target in all
    const int64_t bound = std::min<int64_t>((int64_t)a.target + a.n_seqs,
                                            a.n_seqs * cdiv(longest, a.min_steps));
    a.max_parts = (int32_t)std::max<int64_t>(1, bound);
    if (longest <= a.min_steps) return 0;
    return (size_t)a.max_parts * a.c.n_heads * a.row_blocks * 16 * a.row_tiles *
           (a.c.dim + 2) * sizeof(float);
}

hipError_t launch_attention(const Attention &a, hipStream_t stream)
{
    const int64_t units = cdiv((int64_t)a.max_parts * a.c.n_heads, 8) * 8;
    const dim3 grid((unsigned)(units * a.row_blocks));
    const bool half = a.q.dtype == KVR_DT_FP16;
    hipError_t e;
    switch (a.c.format) {
    case KVR_KV_BF16: e = launch_attention_bf16(a, grid, stream); break;
    case KVR_KV_FP16: e = launch_attention_fp16(a, grid, stream); break;
    case KVR_KV_FP8:
        e = half ? launch_attention_fp8h(a, grid, stream) : launch_attention_fp8(a, grid, stream);
        break;
    default:
        e = half ? launch_attention_fp4h(a, grid, stream) : launch_attention_fp4(a, grid, stream);
    }
    if (e != hipSuccess || a.part_o == nullptr) return e;
    const dim3 joins((unsigned)(a.max_q * a.group), a.c.n_heads, a.n_seqs);
    if (half) combine_kernel<KVR_DT_FP16><<<joins, 256, 0, stream>>>(a, a.c.dim);
    else combine_kernel<KVR_DT_BF16><<<joins, 256, 0, stream>>>(a, a.c.dim);
    return hipGetLastError();
}

}  // namespace kv
}  // namespace kvr
