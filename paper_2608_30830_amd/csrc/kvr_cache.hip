// Rows into and out of the paged KV cache.
//
// Writing quantises as it goes: a block of 32 elements keeps one power of two,
// 2^k with k the smallest exponent for which no code saturates, and 32 codes
// x / 2^k rounded to nearest even in e4m3 or e2m1.  A power of two divides
// exactly, so the code's rounding is the only one.  Keys may be rotated on the
// way, in 32 bits, so a rotated key is rounded once.  A block that holds a NaN
// or an infinity keeps the scale byte 255 and reads as NaN.
//
// Both directions are bound by memory.  A lane holds eight adjacent elements
// (16 bytes of 16-bit input), four lanes a block (its maximum by two quad
// permutes), dim / 8 lanes a row, and consecutive rows are a token's heads.
#include "kvr_kv_device.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kThreads = 256;

struct WriteArgs {
    Cache c;
    Rows k, v;
    Rotary r;
    const int64_t *slots;
    uint32_t rows;       // tokens * heads
    int32_t lane_shift;  // log2 of the lanes of a row
    int *status;
};

enum { kNoRot = 0, kHalf = 1, kInterleaved = 2, kAnyRot = 3 };

// Eight elements from d on of a key row, rotated.
template <int DT, int ROT>
__device__ __forceinline__ void load_rotated(const char *row, int d, const Rotary &r, int64_t pos,
                                             float (&x)[8])
{
#pragma clang fp contract(off)
    constexpr int E = elem_bytes<DT>();
    const int half = r.rot >> 1;
    load8<DT>(row + d * E, x);
    if (ROT == kNoRot || d >= r.rot) return;
    const float *tr = r.t + pos * r.rot;
    if (ROT == kHalf) {
        const bool first = d < half;
        const int i = first ? d : d - half;
        float y[8];
        load8<DT>(row + (first ? d + half : d - half) * E, y);
#pragma unroll
        for (int m = 0; m < 8; m += 4) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(tr + i + m);
            const f32x4 s = *reinterpret_cast<const f32x4 *>(tr + half + i + m);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float t = y[m + n] * (s[n] * r.sign);
                x[m + n] = x[m + n] * c[n] + (first ? -t : t);
            }
        }
    } else if (ROT == kInterleaved) {
        const f32x4 c = *reinterpret_cast<const f32x4 *>(tr + d / 2);
        const f32x4 s = *reinterpret_cast<const f32x4 *>(tr + half + d / 2);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const float a = x[2 * n], b = x[2 * n + 1], sn = s[n] * r.sign;
            x[2 * n] = a * c[n] - b * sn;
            x[2 * n + 1] = b * c[n] + a * sn;
        }
    } else {
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const int e = d + n;
            if (e >= r.rot) break;
            const bool first = r.interleaved ? (e & 1) == 0 : e < half;
            const int i = r.interleaved ? e >> 1 : first ? e : e - half;
            const int o = r.interleaved ? e ^ 1 : first ? e + half : e - half;
            const float t = load1<DT>(row, o) * (tr[half + i] * r.sign);
            x[n] = x[n] * tr[i] + (first ? -t : t);
        }
    }
}

template <int DT, int FMT, int ROT>
__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a)
{
    constexpr int E = elem_bytes<DT>();
    const uint32_t row = blockIdx.x * (uint32_t)(kThreads >> a.lane_shift) +
                         (threadIdx.x >> a.lane_shift);
    const int d = 8 * (threadIdx.x & ((1 << a.lane_shift) - 1));
    if (row >= a.rows || d >= a.c.dim) return;   // whole quads: dim is a multiple of 32
    const uint32_t token = row / (uint32_t)a.c.n_heads;
    const int h = (int)(row - token * (uint32_t)a.c.n_heads);
    const bool key = blockIdx.y == 0;
    const int64_t slot = a.slots[token];
    if (slot < 0) return;
    const int64_t page = slot >> a.c.page_shift;
    int64_t pos = 0;
    bool ok = page < a.c.n_pages;
    if (ROT != kNoRot) {
        pos = a.r.pos[token];
        ok = ok && pos >= 0 && pos < a.r.n_pos;
    }
    if (!ok) {
        if (a.status) *a.status = KVR_E_DOMAIN;
        return;
    }
    const Rows &in = key ? a.k : a.v;
    const char *src = in.p + ((int64_t)token * in.token_stride + (int64_t)h * in.head_stride) * E;
    float x[8];
    if (key) load_rotated<DT, ROT>(src, d, a.r, pos, x);
    else load8<DT>(src + d * E, x);

    const int64_t off = slot & ((1ll << a.c.page_shift) - 1);
    char *dst = (key ? a.c.k : a.c.v) + page * a.c.page_stride + h * a.c.head_stride +
                off * a.c.token_stride;
    if (FMT == KVR_KV_BF16 || FMT == KVR_KV_FP16) {
        store8<FMT == KVR_KV_BF16 ? KVR_DT_BF16 : KVR_DT_FP16>(dst + d * 2, x);
        return;
    }
    uint32_t m = 0;
#pragma unroll
    for (int n = 0; n < 8; ++n) m = max(m, mag_bits(x[n]));
    const uint32_t byte = scale_byte<FMT>(quad_max(m));
    const bool bad = byte == kBadScale;
    // 1 / 2^k: exponent 254 - byte, normal for every byte from 17 to 253
    const float inv = __uint_as_float((254u - (bad ? 127u : byte)) << 23);
#pragma unroll
    for (int n = 0; n < 8; ++n) x[n] = bad ? 0.0f : x[n] * inv;
    if (FMT == KVR_KV_FP8) {
        u32x2 w;
        w[0] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
            x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true);
        w[1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
            x[6], x[7], __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false), true);
        *reinterpret_cast<u32x2 *>(dst + d) = w;
    } else {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.0f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.0f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.0f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.0f, 3);
        *reinterpret_cast<uint32_t *>(dst + d / 2) = w;
    }
    if ((d & 31) == 0) {
        uint8_t *sc = (key ? a.c.ks : a.c.vs) + page * a.c.spage_stride + h * a.c.shead_stride +
                      off * a.c.stoken_stride;
        sc[d >> 5] = (uint8_t)byte;
    }
}

struct ReadArgs {
    Cache c;
    Rows k, v;
    const int64_t *slots;
    uint32_t rows;
    int32_t lane_shift;
    int *status;
};

template <int FMT, int DT>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a)
{
    constexpr int E = elem_bytes<DT>();
    const uint32_t row = blockIdx.x * (uint32_t)(kThreads >> a.lane_shift) +
                         (threadIdx.x >> a.lane_shift);
    const int d = 8 * (threadIdx.x & ((1 << a.lane_shift) - 1));
    if (row >= a.rows || d >= a.c.dim) return;
    const uint32_t token = row / (uint32_t)a.c.n_heads;
    const int h = (int)(row - token * (uint32_t)a.c.n_heads);
    const bool key = blockIdx.y == 0;
    const Rows &out = key ? a.k : a.v;
    char *dst = out.p + ((int64_t)token * out.token_stride + (int64_t)h * out.head_stride + d) * E;
    const int64_t slot = a.slots[token];
    const int64_t page = slot >> a.c.page_shift;
    float x[8];
    if (slot < 0 || page >= a.c.n_pages) {
        if (slot >= 0 && a.status) *a.status = KVR_E_DOMAIN;
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = 0.0f;
        store8<DT>(dst, x);
        return;
    }
    const int64_t off = slot & ((1ll << a.c.page_shift) - 1);
    const char *src = (key ? a.c.k : a.c.v) + page * a.c.page_stride + h * a.c.head_stride +
                      off * a.c.token_stride;
    if (FMT == KVR_KV_BF16 || FMT == KVR_KV_FP16) {
        load8<FMT == KVR_KV_BF16 ? KVR_DT_BF16 : KVR_DT_FP16>(src + d * 2, x);
        store8<DT>(dst, x);
        return;
    }
    const uint8_t *sc = (key ? a.c.ks : a.c.vs) + page * a.c.spage_stride + h * a.c.shead_stride +
                        off * a.c.stoken_stride;
    const float scale = scale_of(sc[d >> 5]);
    u32x2 w;
    if (FMT == KVR_KV_FP8) w = *reinterpret_cast<const u32x2 *>(src + d);
    else w[0] = *reinterpret_cast<const uint32_t *>(src + d / 2);
    // through bfloat16, which holds every value exactly
    uint32_t p[4];
    if (FMT == KVR_KV_FP8) {
        p[0] = codes_to_bf16x2<FMT, 0>(w[0], scale);
        p[1] = codes_to_bf16x2<FMT, 1>(w[0], scale);
        p[2] = codes_to_bf16x2<FMT, 0>(w[1], scale);
        p[3] = codes_to_bf16x2<FMT, 1>(w[1], scale);
    } else {
        p[0] = codes_to_bf16x2<FMT, 0>(w[0], scale);
        p[1] = codes_to_bf16x2<FMT, 1>(w[0], scale);
        p[2] = codes_to_bf16x2<FMT, 2>(w[0], scale);
        p[3] = codes_to_bf16x2<FMT, 3>(w[0], scale);
    }
    if (DT == KVR_DT_BF16) {
        *reinterpret_cast<u32x4 *>(dst) = u32x4{p[0], p[1], p[2], p[3]};
        return;
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) unpack16<KVR_DT_BF16>(p[n], x[2 * n], x[2 * n + 1]);
    store8<DT>(dst, x);
}

int lane_shift(int dim)
{
    int s = 2;
    while ((8 << s) < dim) ++s;
    return s;
}

template <int DT, int FMT>
hipError_t write_rot(const WriteArgs &a, dim3 grid, hipStream_t stream)
{
    int rot = kNoRot;
    if (a.r.t) {
        const bool table = ((uintptr_t)a.r.t & 15) == 0;
        rot = a.r.interleaved ? (table && a.r.rot % 8 == 0 ? kInterleaved : kAnyRot)
                              : (table && a.r.rot % 16 == 0 ? kHalf : kAnyRot);
    }
    switch (rot) {
    case kNoRot: write_kernel<DT, FMT, kNoRot><<<grid, kThreads, 0, stream>>>(a); break;
    case kHalf: write_kernel<DT, FMT, kHalf><<<grid, kThreads, 0, stream>>>(a); break;
    case kInterleaved: write_kernel<DT, FMT, kInterleaved><<<grid, kThreads, 0, stream>>>(a); break;
    default: write_kernel<DT, FMT, kAnyRot><<<grid, kThreads, 0, stream>>>(a); break;
    }
    return hipGetLastError();
}

template <int DT>
hipError_t write_fmt(const WriteArgs &a, dim3 grid, hipStream_t stream)
{
    switch (a.c.format) {
    case KVR_KV_BF16: return write_rot<DT, KVR_KV_BF16>(a, grid, stream);
    case KVR_KV_FP16: return write_rot<DT, KVR_KV_FP16>(a, grid, stream);
    case KVR_KV_FP8: return write_rot<DT, KVR_KV_FP8>(a, grid, stream);
    default: return write_rot<DT, KVR_KV_FP4>(a, grid, stream);
    }
}

template <int FMT>
hipError_t read_out(const ReadArgs &a, int dtype, dim3 grid, hipStream_t stream)
{
    switch (dtype) {
    case KVR_DT_BF16: read_kernel<FMT, KVR_DT_BF16><<<grid, kThreads, 0, stream>>>(a); break;
    case KVR_DT_FP16: read_kernel<FMT, KVR_DT_FP16><<<grid, kThreads, 0, stream>>>(a); break;
    default: read_kernel<FMT, KVR_DT_FP32><<<grid, kThreads, 0, stream>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                              const int64_t *slots, const Rotary &r, int *status,
                              hipStream_t stream)
{
    const WriteArgs a{c, k, v, r, slots, (uint32_t)(tokens * c.n_heads), lane_shift(c.dim), status};
    const dim3 grid((unsigned)cdiv(a.rows, kThreads >> a.lane_shift), 2);
    switch (k.dtype) {
    case KVR_DT_BF16: return write_fmt<KVR_DT_BF16>(a, grid, stream);
    case KVR_DT_FP16: return write_fmt<KVR_DT_FP16>(a, grid, stream);
    default: return write_fmt<KVR_DT_FP32>(a, grid, stream);
    }
}

hipError_t launch_cache_read(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                             const int64_t *slots, int *status, hipStream_t stream)
{
    const ReadArgs a{c, k, v, slots, (uint32_t)(tokens * c.n_heads), lane_shift(c.dim), status};
    const dim3 grid((unsigned)cdiv(a.rows, kThreads >> a.lane_shift), 2);
    switch (c.format) {
    case KVR_KV_BF16: return read_out<KVR_KV_BF16>(a, k.dtype, grid, stream);
    case KVR_KV_FP16: return read_out<KVR_KV_FP16>(a, k.dtype, grid, stream);
    case KVR_KV_FP8: return read_out<KVR_KV_FP8>(a, k.dtype, grid, stream);
    default: return read_out<KVR_KV_FP4>(a, k.dtype, grid, stream);
    }
}

}  // namespace kv
}  // namespace kvr
