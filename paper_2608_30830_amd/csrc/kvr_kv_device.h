// Device helpers of the KV-cache kernels: rows of eight elements, 16-bit
// conversions, block scales.
#pragma once

#include "kvr_kv.h"

namespace kvr {
namespace kv {

// The block's number in a launch by grid_of; those beyond its last one are the caller's to end.
__device__ __forceinline__ uint32_t block_of_grid() { return blockIdx.z * kMaxGrid + blockIdx.x; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b)
{
    f16x2 r = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, r);
}
template <int DT>
__device__ __forceinline__ uint32_t pack16(float a, float b)
{
    return DT == KVR_DT_BF16 ? pack_bf16(a, b) : pack_f16(a, b);
}
template <int DT>
__device__ __forceinline__ void unpack16(uint32_t x, float &a, float &b)
{
    if (DT == KVR_DT_BF16) {
        a = __uint_as_float(x << 16);
        b = __uint_as_float(x & 0xffff0000u);
    } else {
        const f16x2 r = __builtin_bit_cast(f16x2, x);
        a = (float)r[0];
        b = (float)r[1];
    }
}

template <int DT>
__device__ __forceinline__ float load1(const char *p, int64_t i)
{
    if (DT == KVR_DT_FP32) return reinterpret_cast<const float *>(p)[i];
    if (DT == KVR_DT_BF16)
        return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(p)[i] << 16);
    return (float)reinterpret_cast<const _Float16 *>(p)[i];
}
template <int DT>
__device__ __forceinline__ void store1(char *p, int64_t i, float x)
{
    if (DT == KVR_DT_FP32) reinterpret_cast<float *>(p)[i] = x;
    else if (DT == KVR_DT_BF16) reinterpret_cast<__bf16 *>(p)[i] = (__bf16)x;
    else reinterpret_cast<_Float16 *>(p)[i] = (_Float16)x;
}

// 16 bytes; Stream: past the caches.
template <bool Stream = false, class T>
__device__ __forceinline__ void store16(T *p, T x)
{
    if (Stream) __builtin_nontemporal_store(x, p);
    else *p = x;
}

// Eight adjacent elements from a 16-byte aligned address.
template <int DT>
__device__ __forceinline__ void load8(const char *p, float (&x)[8])
{
    if (DT == KVR_DT_FP32) {
        const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0];
        const f32x4 b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack16<DT>(a[i], x[2 * i], x[2 * i + 1]);
    }
}
template <int DT, bool Stream = false>
__device__ __forceinline__ void store8(char *p, const float (&x)[8])
{
    if (DT == KVR_DT_FP32) {
        store16<Stream>(reinterpret_cast<f32x4 *>(p), f32x4{x[0], x[1], x[2], x[3]});
        store16<Stream>(reinterpret_cast<f32x4 *>(p) + 1, f32x4{x[4], x[5], x[6], x[7]});
    } else {
        store16<Stream>(reinterpret_cast<u32x4 *>(p),
                        u32x4{pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]),
                              pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7])});
    }
}

template <int DT>
constexpr int elem_bytes()
{
    return DT == KVR_DT_FP32 ? 4 : 2;
}

// The number that a scale byte stands for: 2^(byte - 127).  255 gives an
// infinity's bits, which the conversions below read as NaN, as they do every
// scale of that exponent.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes to 16-bit or 32-bit values.  The conversions take the scale's
// exponent, and e4m3 and e2m1 values times a power of two are exact in
// bfloat16 (and in 32 bits).
template <int FMT, int HALF>
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t codes, float scale)
{
    if (FMT == KVR_KV_FP8)
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HALF != 0));
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, HALF));
}

__device__ __forceinline__ uint32_t mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Largest magnitude (as bits: NaN > infinity > numbers) over the four lanes
// that hold a block of 32.
__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true);
    x = x > y ? x : y;
    y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true);
    return x > y ? x : y;
}

// Scale byte of a block whose largest magnitude has these bits: the smallest
// exponent k with magnitude <= M 2^k, M = 448 (mantissa 1.75, exponent 8) or 6
// (1.5, 2), so that no code saturates; a mantissa beyond M's carries into the
// exponent.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax)
{
    constexpr uint32_t over = FMT == KVR_KV_FP8 ? 0x7fffffu - 0x600000u : 0x7fffffu - 0x400000u;
    constexpr int top = FMT == KVR_KV_FP8 ? 8 : 2;
    if (amax >= 0x7f800000u) return kBadScale;
    const int e = (int)((amax + over) >> 23) - top;
    return (uint32_t)(e > kMinExp + 127 ? e : kMinExp + 127);
}

}  // namespace kv
}  // namespace kvr
