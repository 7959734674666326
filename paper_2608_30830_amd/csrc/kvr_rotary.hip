// Rotary positions.  Pair i of a row (of rot / 2) turns by the angle p w_i of
// its position p:
//   a' = a cos - b sin,   b' = b cos + a sin
// with a, b = x[i], x[i + rot/2] (half layout) or x[2i], x[2i + 1]
// (interleaved); elements from rot on are copied.  The adjoint (the gradient
// with respect to x) turns by the negative angle.  cos and sin come from a
// table, times the table's magnitude.
//
// The operator moves 2 * tokens * heads * dim elements and computes three
// operations for each, so memory bounds it: a lane takes both halves of eight
// pairs (two 16-byte loads in 16-bit types), which also makes it safe in place,
// and up to four heads of its token, so that their loads are in flight together
// and a table row is read once for them.  32,768 tokens of 32 heads of 128 in 16 bits:
// 101 us (5.5 TB/s; a copy of that size reaches 5.1 to 5.5), 90 when the inputs are in
// the last cache.
#include "kvr_kv_device.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kThreads = 256;

// One thread per (position, pair).  The phase is formed in 64 bits: at position
// 131,072 a 32-bit one would be off by 2^-8.
__global__ __launch_bounds__(kThreads) void table_kernel(Freqs f, double magnitude, int half,
                                                         int64_t total, float *t)
{
    const int64_t i = (int64_t)block_of_grid() * kThreads + threadIdx.x;
    if (i >= total) return;
    const int64_t pos = i / half;
    const int j = (int)(i - pos * half);
    double s, c;
    sincos((double)pos * f.w[j], &s, &c);
    float *row = t + pos * 2 * half;
    row[j] = (float)(magnitude * c);
    row[half + j] = (float)(magnitude * s);
}

struct RotaryArgs {
    Rows x, out;
    Rotary r;
    uint32_t tokens;
    int heads, dim, units, rot_units, head_groups, tokens_per_block;
    int *status;
};

// The products are rounded one by one (no fused multiply-add), so that every
// path that rotates gives the same bits.
__device__ __forceinline__ void turn(float &a, float &b, float c, float s)
{
#pragma clang fp contract(off)
    const float y = a * c - b * s;
    b = b * c + a * s;
    a = y;
}

template <int DT, bool IL, int HPT, bool Stream = false>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    constexpr int E = elem_bytes<DT>();
    const int lanes = a.head_groups * a.units;
    const int work = a.tokens_per_block * lanes;
    const int half = a.r.rot >> 1;
    for (int i = threadIdx.x; i < work; i += kThreads) {
        const int tb = i / lanes, rest = i - tb * lanes;
        const int hg = rest / a.units, u = rest - hg * a.units;
        const uint32_t token = block_of_grid() * (uint32_t)a.tokens_per_block + tb;
        if (token >= a.tokens) return;
        const char *xr = a.x.p + (int64_t)token * a.x.token_stride * E;
        char *yr = a.out.p + (int64_t)token * a.out.token_stride * E;
        if (u >= a.rot_units) {   // the part that keeps its place
            const int d = a.r.rot + 8 * (u - a.rot_units);
#pragma unroll
            for (int j = 0; j < HPT; ++j) {
                const int h = hg + j * a.head_groups;
                if (h >= a.heads) break;
                float v[8];
                load8<DT>(xr + ((int64_t)h * a.x.head_stride + d) * E, v);
                store8<DT, Stream>(yr + ((int64_t)h * a.out.head_stride + d) * E, v);
            }
            continue;
        }
        int64_t pos = a.r.pos[token];
        if (pos < 0 || pos >= a.r.n_pos) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            pos = 0;
        }
        const int p = IL ? 4 * u : 8 * u;   // first pair of the unit
        constexpr int NP = IL ? 4 : 8;
        const float *tr = a.r.t + pos * a.r.rot + p;
        float x0[HPT][8], x1[HPT][8];
        const int d0 = IL ? 8 * u : 8 * u;
#pragma unroll
        for (int j = 0; j < HPT; ++j) {
            const int h = hg + j * a.head_groups;
            if (h < a.heads) {
                const char *q = xr + ((int64_t)h * a.x.head_stride + d0) * E;
                load8<DT>(q, x0[j]);
                if (!IL) load8<DT>(q + half * E, x1[j]);
            }
        }
        float c[NP], s[NP];
#pragma unroll
        for (int k = 0; k < NP; k += 4) {
            const f32x4 cc = *reinterpret_cast<const f32x4 *>(tr + k);
            const f32x4 ss = *reinterpret_cast<const f32x4 *>(tr + half + k);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                c[k + m] = cc[m];
                s[k + m] = ss[m] * a.r.sign;
            }
        }
#pragma unroll
        for (int j = 0; j < HPT; ++j) {
            const int h = hg + j * a.head_groups;
            if (h >= a.heads) break;
            char *q = yr + ((int64_t)h * a.out.head_stride + d0) * E;
            if (IL) {
#pragma unroll
                for (int k = 0; k < 4; ++k) turn(x0[j][2 * k], x0[j][2 * k + 1], c[k], s[k]);
                store8<DT, Stream>(q, x0[j]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) turn(x0[j][k], x1[j][k], c[k], s[k]);
                store8<DT, Stream>(q, x0[j]);
                store8<DT, Stream>(q + half * E, x1[j]);
            }
        }
    }
}

// Rows that eight elements at a time do not fit (rot not a multiple of 16, or of
// 8 interleaved; strides or addresses off 16 bytes): a pair, or a copied
// element, at a time.
template <int DT>
__global__ __launch_bounds__(kThreads) void rotary_pairs_kernel(RotaryArgs a)
{
    constexpr int E = elem_bytes<DT>();
    const int half = a.r.rot >> 1;
    const int lanes = a.heads * a.units;
    const int work = a.tokens_per_block * lanes;
    for (int i = threadIdx.x; i < work; i += kThreads) {
        const int tb = i / lanes, rest = i - tb * lanes;
        const int h = rest / a.units, u = rest - h * a.units;
        const uint32_t token = block_of_grid() * (uint32_t)a.tokens_per_block + tb;
        if (token >= a.tokens) return;
        const char *x = a.x.p + ((int64_t)token * a.x.token_stride + (int64_t)h * a.x.head_stride) * E;
        char *y = a.out.p + ((int64_t)token * a.out.token_stride + (int64_t)h * a.out.head_stride) * E;
        if (u >= half) {
            const int d = a.r.rot + (u - half);
            store1<DT>(y, d, load1<DT>(x, d));
            continue;
        }
        int64_t pos = a.r.pos[token];
        if (pos < 0 || pos >= a.r.n_pos) {
            if (a.status) *a.status = KVR_E_DOMAIN;
            pos = 0;
        }
        const float *tr = a.r.t + pos * a.r.rot + u;
        const int i0 = a.r.interleaved ? 2 * u : u, i1 = a.r.interleaved ? 2 * u + 1 : u + half;
        float v0 = load1<DT>(x, i0), v1 = load1<DT>(x, i1);
        turn(v0, v1, tr[0], tr[half] * a.r.sign);
        store1<DT>(y, i0, v0);
        store1<DT>(y, i1, v1);
    }
}

bool rows_aligned(const Rows &r)
{
    const int64_t e = r.dtype == KVR_DT_FP32 ? 4 : 2;
    return ((uintptr_t)r.p & 15) == 0 && (r.token_stride * e & 15) == 0 &&
           (r.head_stride * e & 15) == 0;
}

template <int DT>
hipError_t launch(RotaryArgs &a, bool copy_tail, hipStream_t stream)
{
    const int rot = a.r.rot;
    const bool il = a.r.interleaved != 0;
    const bool wide = rows_aligned(a.x) && rows_aligned(a.out) && a.dim % 8 == 0 &&
                      rot % (il ? 8 : 16) == 0 && ((uintptr_t)a.r.t & 15) == 0;
    // four heads a lane once that still leaves 2,048 waves or more
    int hpt = 1;
    if (wide) {
        a.rot_units = il ? rot / 8 : rot / 16;
        a.units = a.rot_units + (copy_tail ? (a.dim - rot) / 8 : 0);
        if (a.heads >= 4 && (int64_t)a.tokens * a.heads * a.units >= 4 * 2048 * 64) hpt = 4;
        a.head_groups = (a.heads + hpt - 1) / hpt;
    } else {
        a.rot_units = rot / 2;
        a.units = rot / 2 + (copy_tail ? a.dim - rot : 0);
        a.head_groups = a.heads;
    }
    const int lanes = a.head_groups * a.units;
    a.tokens_per_block = lanes >= kThreads ? 1 : kThreads / lanes;
    const dim3 grid = grid_of(cdiv(a.tokens, a.tokens_per_block));
    const bool large = hpt == 4 && streams((int64_t)a.tokens * a.heads * a.dim, a.dim, DT);
    if (!wide) rotary_pairs_kernel<DT><<<grid, kThreads, 0, stream>>>(a);
    else if (il && large) rotary_kernel<DT, true, 4, DT != KVR_DT_FP32><<<grid, kThreads, 0, stream>>>(a);
    else if (il && hpt == 4) rotary_kernel<DT, true, 4><<<grid, kThreads, 0, stream>>>(a);
    else if (il) rotary_kernel<DT, true, 1><<<grid, kThreads, 0, stream>>>(a);
    else if (large) rotary_kernel<DT, false, 4, DT != KVR_DT_FP32><<<grid, kThreads, 0, stream>>>(a);
    else if (hpt == 4) rotary_kernel<DT, false, 4><<<grid, kThreads, 0, stream>>>(a);
    else rotary_kernel<DT, false, 1><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary_table(const Freqs &f, double magnitude, int rot, int64_t n_pos,
                               float *table, hipStream_t stream)
{
    const int half = rot / 2;
    const int64_t total = n_pos * half;
    table_kernel<<<grid_of(cdiv(total, kThreads)), kThreads, 0, stream>>>(f, magnitude, half,
                                                                               total, table);
    return hipGetLastError();
}

hipError_t launch_rotary(const Rows &x, const Rows &out, int64_t tokens, int heads, int dim,
                         const Rotary &r, int *status, hipStream_t stream)
{
    RotaryArgs a{};
    a.x = x;
    a.out = out;
    a.r = r;
    a.tokens = (uint32_t)tokens;
    a.heads = heads;
    a.dim = dim;
    a.status = status;
    const bool in_place = x.p == out.p && x.token_stride == out.token_stride &&
                          x.head_stride == out.head_stride;
    switch (x.dtype) {
    case KVR_DT_BF16: return launch<KVR_DT_BF16>(a, !in_place, stream);
    case KVR_DT_FP16: return launch<KVR_DT_FP16>(a, !in_place, stream);
    default: return launch<KVR_DT_FP32>(a, !in_place, stream);
    }
}

}  // namespace kv
}  // namespace kvr
