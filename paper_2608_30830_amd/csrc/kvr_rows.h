// Eight elements of a row a lane: loaded as they lie, rotated, put into a cache's
// format and taken out of it.  For the kernels that move rows into and out of caches.
#pragma once

#include "kvr_kv_device.h"

namespace kvr {
namespace kv {
namespace {

enum { kNoRot = 0, kHalf = 1, kInterleaved = 2, kAnyRot = 3 };

// Eight elements as they lie in memory.
template <int DT>
struct Raw {
    u32x4 w[DT == KVR_DT_FP32 ? 2 : 1];
    __device__ __forceinline__ void load(const char *p)
    {
        w[0] = reinterpret_cast<const u32x4 *>(p)[0];
        if (DT == KVR_DT_FP32) w[DT == KVR_DT_FP32] = reinterpret_cast<const u32x4 *>(p)[1];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == KVR_DT_FP32) {
                x[i] = __uint_as_float(w[0][i]);
                x[4 + i] = __uint_as_float(w[DT == KVR_DT_FP32][i]);
            } else {
                unpack16<DT>(w[0][i], x[2 * i], x[2 * i + 1]);
            }
        }
    }
};

// What a lane needs to rotate its eight elements from d on, for all heads of a token.
template <int ROT>
struct Turn {
    float c[ROT == kHalf ? 8 : 4], s[ROT == kHalf ? 8 : 4];
    bool on, first;
    __device__ __forceinline__ void load(const Rotary &r, int64_t pos, int d)
    {
        const int half = r.rot >> 1;
        on = ROT != kNoRot && d < r.rot;
        first = d < half;
        if (!on || ROT == kAnyRot) return;
        const int i = ROT == kInterleaved ? d / 2 : first ? d : d - half;
        const float *tr = r.t + pos * r.rot + i;
        constexpr int N = ROT == kHalf ? 8 : 4;
#pragma unroll
        for (int m = 0; m < N; m += 4) {
            const f32x4 cc = *reinterpret_cast<const f32x4 *>(tr + m);
            const f32x4 ss = *reinterpret_cast<const f32x4 *>(tr + half + m);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                c[m + n] = cc[n];
                s[m + n] = ss[n] * r.sign;
            }
        }
    }
};

// x: the eight elements from d on; y: their partners (half layout).
template <int DT, int ROT>
__device__ __forceinline__ void rotate(const Turn<ROT> &t, const char *row, int d, const Rotary &r,
                                       int64_t pos, const Raw<DT> &partner, float (&x)[8])
{
#pragma clang fp contract(off)
    if (!t.on) return;
    if constexpr (ROT == kHalf) {
        float y[8];
        partner.get(y);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float z = y[n] * t.s[n];
            x[n] = x[n] * t.c[n] + (t.first ? -z : z);
        }
    } else if constexpr (ROT == kInterleaved) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const float a = x[2 * n], b = x[2 * n + 1];
            x[2 * n] = a * t.c[n] - b * t.s[n];
            x[2 * n + 1] = b * t.c[n] + a * t.s[n];
        }
    } else if constexpr (ROT == kAnyRot) {
        const int half = r.rot >> 1;
        const float *tr = r.t + pos * r.rot;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const int e = d + n;
            if (e >= r.rot) break;
            const bool first = r.interleaved ? (e & 1) == 0 : e < half;
            const int i = r.interleaved ? e >> 1 : first ? e : e - half;
            const int o = r.interleaved ? e ^ 1 : first ? e + half : e - half;
            const float z = load1<DT>(row, o) * (tr[half + i] * r.sign);
            x[n] = x[n] * tr[i] + (first ? -z : z);
        }
    }
}

// Eight elements from d on into the row at dst, with the block's scale byte at sc.
template <int FMT>
__device__ __forceinline__ void put_row(char *dst, uint8_t *sc, int d, float (&x)[8])
{
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
    if ((d & 31) == 0) sc[d >> 5] = (uint8_t)byte;
}

// Eight elements of a row as loaded.
template <int FMT>
struct Codes {
    static constexpr bool Quant = FMT == KVR_KV_FP8 || FMT == KVR_KV_FP4;
    uint32_t w[FMT == KVR_KV_FP4 ? 1 : FMT == KVR_KV_FP8 ? 2 : 4];
    uint32_t scale;
    __device__ __forceinline__ void load(const char *row, const uint8_t *sc, int d)
    {
        if constexpr (FMT == KVR_KV_FP4) {
            w[0] = *reinterpret_cast<const uint32_t *>(row + d / 2);
        } else if constexpr (FMT == KVR_KV_FP8) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(row + d);
            w[0] = x[0], w[1] = x[1];
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(row + 2 * d);
            w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
        }
        if (Quant) scale = sc[d >> 5];
    }
    // As 16-bit values: the cache's own, or bfloat16, which holds every code's value.
    __device__ __forceinline__ void get(uint32_t (&p)[4]) const
    {
        if constexpr (FMT == KVR_KV_FP8) {
            const float s = scale_of(scale);
            p[0] = codes_to_bf16x2<FMT, 0>(w[0], s);
            p[1] = codes_to_bf16x2<FMT, 1>(w[0], s);
            p[2] = codes_to_bf16x2<FMT, 0>(w[1], s);
            p[3] = codes_to_bf16x2<FMT, 1>(w[1], s);
        } else if constexpr (FMT == KVR_KV_FP4) {
            const float s = scale_of(scale);
            p[0] = codes_to_bf16x2<FMT, 0>(w[0], s);
            p[1] = codes_to_bf16x2<FMT, 1>(w[0], s);
            p[2] = codes_to_bf16x2<FMT, 2>(w[0], s);
            p[3] = codes_to_bf16x2<FMT, 3>(w[0], s);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = w[i];
        }
    }
};

// How the rotation of a call can be done: eight elements a lane at a time, or any.
inline int rotation_kind(const Rotary &r)
{
    if (!r.t) return kNoRot;
    const bool table = ((uintptr_t)r.t & 15) == 0;
    if (table && !r.interleaved && r.rot % 16 == 0) return kHalf;
    if (table && r.interleaved && r.rot % 8 == 0) return kInterleaved;
    return kAnyRot;
}

}  // namespace
}  // namespace kv
}  // namespace kvr
