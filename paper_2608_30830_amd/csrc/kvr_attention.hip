// Attention over the paged cache: the launch plan, and the kernel that joins the
// parts of sequences that were cut.
#include <algorithm>

#include "kvr_parts.h"

namespace kvr {
namespace kv {
namespace {

// Joins the parts of rows.  A row has dim / 4 lanes times Groups groups of parts: each
// group goes through its share of the parts, four at a time, with a running
// maximum, then the groups are added in order.  With many rows one group does, with
// few several keep more loads in flight, and with many parts of few rows as many as a
// block holds (a read of four parts takes about a microsecond, however few rows).
template <int QT, int Groups, int Threads>
__global__ __launch_bounds__(Threads) void combine_kernel(Attention a)
{
    constexpr int N = Groups > 1 ? Threads : 1;
    __shared__ __align__(16) float so[4 * N];
    __shared__ float sl[N], sm[N], sw[N];
    const int dim = a.c.dim, cols = dim / 4;
    const int per_row = cols * Groups;
    const int rows_per_block = Threads / per_row;
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
    int len, nq, q0;
    sequence(a, b, len, nq, q0);
    const int rows = nq * a.group;
    if ((int)blockIdx.x * rows_per_block >= rows) return;
    Lane x = lane_sequence(a, 0);
    const int per = part_steps(a, x);
    const int parts = parts_of(steps_of(len, nq), per);
    if (parts <= 1) return;
    int64_t base = 0;   // items before this sequence's
    for (int b0 = 0; b0 < b; b0 += 64) {
        if (b0) x = lane_sequence(a, b0);
        base += wave_total(b0 + lane < b ? parts_of(x.steps, per) * x.rbs : 0);
    }
    const int local = threadIdx.x / per_row, rest = threadIdx.x - local * per_row;
    const int grp = rest / cols, c = rest - grp * cols;
    const int row = blockIdx.x * rows_per_block + local;
    const bool live = local < rows_per_block && row < rows;
    const int rb = row / a.block_rows, rr = row - rb * a.block_rows;
    const int nrb = row_blocks_of(a, nq);
    if (!planned(a, base, parts, nrb)) {   // left out (every wave agrees)
        if (a.status) *a.status = KVR_E_DOMAIN;
        return;
    }
    f32x4 acc = {0, 0, 0, 0};
    float sum = 0.0f, norm = 0.0f, top = kLowest;
    if (live) {
        const int64_t first = ((base + rb) * a.c.n_heads + h) * a.block_rows + rr;
        const int64_t next = (int64_t)nrb * a.c.n_heads * a.block_rows;   // cells from part to part
        const float4 *ml = a.part_ml + first;
        const float *o = a.part_o + first * dim + 4 * c;
        for (int p = grp; p < parts; p += 4 * Groups) {
            float4 m[4];   // maximum, sum of the weights, of the rounded ones
            f32x4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t at = min(p + k * Groups, parts - 1) * next;
                m[k] = ml[at];
                v[k] = *reinterpret_cast<const f32x4 *>(o + at * dim);
            }
            float t = top;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (p + k * Groups < parts) t = fmaxf(t, m[k].x);
            const float f = __builtin_amdgcn_exp2f(top - t);
            acc *= f;
            sum *= f;
            norm *= f;
            top = t;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (p + k * Groups < parts) {
                    const float w = __builtin_amdgcn_exp2f(m[k].x - t);
                    sum += w * m[k].y;
                    norm += w * m[k].z;
                    acc += w * v[k];
                }
        }
    }
    if constexpr (Groups > 1) {
        if (live) {
            *reinterpret_cast<f32x4 *>(so + 4 * threadIdx.x) = acc;
            sl[threadIdx.x] = sum;
            sm[threadIdx.x] = top;
            sw[threadIdx.x] = norm;
        }
        __syncthreads();
        if (!live || grp != 0) return;
        float t = top;
#pragma unroll
        for (int p = 1; p < Groups; ++p) t = fmaxf(t, sm[threadIdx.x + p * cols]);
        float f = __builtin_amdgcn_exp2f(top - t);
        acc *= f;
        sum *= f;
        norm *= f;
        top = t;
#pragma unroll
        for (int p = 1; p < Groups; ++p) {
            const int at = threadIdx.x + p * cols;
            f = __builtin_amdgcn_exp2f(sm[at] - t);
            acc += f * *reinterpret_cast<const f32x4 *>(so + 4 * at);
            sum += f * sl[at];
            norm += f * sw[at];
        }
    }
    if (!live) return;
    const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
    const int i0 = row / a.group;
    const int head = h * a.group + (row - i0 * a.group);
    uint32_t *y = reinterpret_cast<uint32_t *>(
        a.out.p + ((int64_t)(q0 + i0) * a.out.token_stride + (int64_t)head * a.out.head_stride + 4 * c) * 2);
    *reinterpret_cast<u32x2 *>(y) = u32x2{pack16<QT>(acc[0] * inv, acc[1] * inv),
                                          pack16<QT>(acc[2] * inv, acc[3] * inv)};
    if (c == 0 && a.lse)
        a.lse[(int64_t)(q0 + i0) * a.q_heads + head] =
            sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int QT>
hipError_t launch_combine(const Attention &a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.max_q * a.group;
    const bool many = rows * a.c.n_heads * a.n_seqs >= 4096;
    const bool narrow = a.c.dim <= 128;
    // Many parts of few sequences: a block of 1,024 (one sequence of 90,196 tokens in 4 bits and
    // one KV head, 470 parts: 24.5 -> 18.7 us a call; with 96 parts of 56 rows 73 -> 75).
    const int64_t parts = std::min<int64_t>(a.target / a.n_seqs, cdiv(a.max_kv, kStep) / a.min_steps);
    const bool deep = !many && parts > 128;
    const int threads = deep ? 1024 : 256;
    const int groups = many ? 1 : (narrow ? 8 : 4) * (threads / 256);   // at most all lanes a row
    const dim3 grid((unsigned)cdiv(rows, threads / (a.c.dim / 4 * groups)), a.c.n_heads, a.n_seqs);
    if (many) combine_kernel<QT, 1, 256><<<grid, 256, 0, stream>>>(a);
    else if (deep && narrow) combine_kernel<QT, 32, 1024><<<grid, 1024, 0, stream>>>(a);
    else if (deep) combine_kernel<QT, 16, 1024><<<grid, 1024, 0, stream>>>(a);
    else if (narrow) combine_kernel<QT, 8, 256><<<grid, 256, 0, stream>>>(a);
    else combine_kernel<QT, 4, 256><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// Blocks that the parts are planned for, of all heads: what is resident at once (two
// blocks on each of 256 CUs, three where 64 rows share tokens), so that equal parts
// end together; twice that where each block has 128 rows, because there the rows of
// ragged sequences fill blocks unevenly (trees of 17 to 64 tokens over 2,048 to 32,768:
// 364 us planned for 512, 350 for 1,024, 344 for 2,048; 512 rows of each sequence over
// 16,384 tokens: 650, 671, 695).
constexpr int kSlots = 512;
constexpr int kShortSteps = 16;    // 512 tokens

}  // namespace

size_t plan_attention(Attention &a)
{
    const int64_t rows = (int64_t)a.max_q * a.group;
    const int64_t longest = cdiv(a.max_kv, kStep);
    // Up to 16 rows: every wave has them all, and a share of the cached tokens.  Up to 32 the
    // same with two row tiles, where registers allow (heads up to 128).  Beyond, waves
    // share the tokens through LDS (56 rows over 131,071 tokens in 4 bits: 66 us against
    // 74 with two row tiles a wave).
    const bool narrow = a.c.dim <= 128;
    a.shared = rows > (narrow ? 32 : 16);
    // (33 to 64 rows in two waves of two tiles, which read half as much LDS: 79 us against 74.)
    a.row_tiles = rows <= 16 || !narrow || (rows > 32 && rows <= 64) ? 1 : 2;
    a.waves = 4;
    // A part's outputs (32 bits) are written and read again: of 128 rows they are worth 8 steps
    // of 16-bit cache (24 sequences of 63 to 184 tokens, 63 new ones, 8 queries a head: 50 us in
    // parts of four steps, 31 in parts of 16).
    a.min_steps = a.shared ? 8 * a.row_tiles : a.waves;
    int slots = kSlots;
    if (a.shared) slots = a.row_tiles > 1 ? 2 * kSlots : kSlots * 3 / 2;
    // Short sequences: no parts, so that one launch does, and eight waves a block while the
    // blocks are not more than the CUs.  (Bfloat16, 8 heads of 128, us a call against parts: one
    // sequence of 500 tokens 10.6, 12.0; of 1,000 14.7, 11.8; 32 of 500 16.0, 20.9; of 1,000
    // 24.1, 28.7; 128 of 2,000 179, 184; 400 of 50 to 2,000 171, 203: where sequences are many,
    // finding the parts and joining them is not free.  With 24 rows a head in 8 bits: one of 500 tokens
    // 11.3, 12.8; 32 of 500 13.6, 19.0; 200 of 500 54, 81; 200 of 2,000 180, 208.)
    const int64_t heads = (int64_t)a.n_seqs * a.c.n_heads;
    if (!a.shared && longest <= kShortSteps * (heads >= 1024 ? 4 : heads >= 128 ? 2 : 1)) {
        a.waves = rows <= 16 && heads <= 256 ? 8 : 4;
        a.min_steps = (int32_t)longest;
    }
    a.block_rows = 16 * a.row_tiles * (a.shared ? a.waves : 1);
    a.target = std::max(1, slots / a.c.n_heads);
    // Row blocks of all sequences; the nearest whole number to steps / part parts of each,
    // part = total / target or min_steps.
    const int64_t blocks = std::min<int64_t>((int64_t)a.n_seqs * cdiv(rows, a.block_rows),
                                             a.n_queries * a.group / a.block_rows + a.n_seqs);
    // (at most 2^30 launched blocks: 2^12 sequences x 2^24 query heads and tokens / 64 rows)
    a.max_items = (int32_t)std::max<int64_t>(
        1, std::min(a.target + blocks, blocks * cdiv(longest, a.min_steps)));
    a.direct = 0;
    if (longest <= a.min_steps) {
        // Nothing is cut: a block knows its sequence from its number, and its first pages are
        // looked up beside the lengths.  Sequences that do not fill their room leave blocks
        // without work.
        const int64_t room = cdiv(rows, a.block_rows);
        if (a.max_pages > 0 && (room == 1 || a.n_seqs * room <= 2 * kSlots)) {
            a.direct = (int32_t)room;
            a.max_items = (int32_t)std::max<int64_t>(1, a.n_seqs * room);
        }
        return 0;
    }
    return (size_t)a.max_items * a.c.n_heads * a.block_rows * (a.c.dim + 4) * sizeof(float);
}

hipError_t launch_attention(const Attention &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.max_items * a.c.n_heads));
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
    return half ? launch_combine<KVR_DT_FP16>(a, stream) : launch_combine<KVR_DT_BF16>(a, stream);
}

}  // namespace kv
}  // namespace kvr
