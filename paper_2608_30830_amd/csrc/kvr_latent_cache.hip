// Rows into and out of the latent cache.
//
// Writing a row: the latent c, with a norm c_i w_i / sqrt(mean(c^2) + eps), and the shared
// key, rotated; in 32 bits, rounded once by the cache's format (blocks of 32 with a power
// of two, as the cache of keys and values).  Memory bounds both directions.  A lane holds
// eight adjacent elements, rank / 8 lanes a latent; a wave of large calls has four
// rows, so that their loads are in flight together, and then takes all their shared keys, which
// fill half of its lanes, in one pass.  32,749 rows of 512 + 64 elements, bfloat16 with a norm to
// codes of 8 bits: written in 19.5 us (57 MB, 2.9 TB/s; the last cache holds part of the input), with eight
// rows a wave in 21.4; read back in 12.0 us (4.7 TB/s).
#include "kvr_dpp.h"
#include "kvr_latent.h"
#include "kvr_rows.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kThreads = 256;

// Sum over N adjacent lanes (a power of two), the same bits in each of them.
template <int N>
__device__ __forceinline__ float lanes_sum(float x)
{
    // 16 lanes by moves within their row, then rows 16 and 32 apart
    x += dpp_move<0xB1, 0xf>(x, 0);   // quads: 1, 0, 3, 2
    x += dpp_move<0x4E, 0xf>(x, 0);   // 2, 3, 0, 1
    x += dpp_move<0x141, 0xf>(x, 0);  // mirrored in eight
    x += dpp_move<0x140, 0xf>(x, 0);  // and in sixteen
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    if (N == 32) return x;
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Where a token's row goes, or nullptr.
struct Place {
    char *row;
    uint8_t *scale;
};
template <int FMT>
__device__ __forceinline__ Place place(const Latents &c, int64_t slot)
{
    const int64_t page = slot >> c.page_shift;
    const int64_t off = slot & ((1ll << c.page_shift) - 1);
    return Place{c.rows + page * c.page_stride + off * c.token_stride,
                 FMT == KVR_KV_FP8 ? c.scale + page * c.spage_stride + off * c.stoken_stride : nullptr};
}

// Whether a token is written: its slot is in the pool and its position in the table.
template <int ROT>
__device__ __forceinline__ bool live(const LatentWrite &a, uint32_t token, int64_t &slot, int64_t &pos)
{
    slot = a.slots[token];
    pos = ROT != kNoRot ? a.r.pos[token] : 0;
    if (slot < 0) return false;
    if (slot >> a.c.page_shift >= a.c.n_pages || (ROT != kNoRot && (pos < 0 || pos >= a.r.n_pos))) {
        if (a.status) *a.status = KVR_E_DOMAIN;
        return false;
    }
    return true;
}

// A wave has T tokens.
template <int DT, int FMT, int ROT, int RANK, int T>
__global__ __launch_bounds__(kThreads) void latent_write_kernel(LatentWrite a)
{
    constexpr int E = elem_bytes<DT>();
    constexpr int Lanes = RANK / 8, PerPass = 64 / Lanes;   // of a latent; latents of a pass
    constexpr int Passes = (T + PerPass - 1) / PerPass;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t first = ((uint64_t)block_of_grid() * (kThreads / 64) + (threadIdx.x >> 6)) * T;
    if (first >= a.tokens) return;
    const uint32_t left = min((uint32_t)T, (uint32_t)(a.tokens - first));
    const uint32_t t0 = (uint32_t)first;
    const int d = 8 * (int)(lane % Lanes);
    Raw<DT> x[Passes];
#pragma unroll
    for (int i = 0; i < Passes; ++i) {
        const uint32_t t = i * PerPass + lane / Lanes;
        if (t < left) x[i].load(a.latent.p + ((int64_t)(t0 + t) * a.latent.token_stride + d) * E);
    }
    float w[8];
    if (a.norm) load8<DT>(a.norm + d * E, w);
#pragma unroll
    for (int i = 0; i < Passes; ++i) {
        const uint32_t t = i * PerPass + lane / Lanes;
        if (t >= left) continue;   // whole groups of Lanes lanes
        float y[8];
        x[i].get(y);
        if (a.norm) {
            float s = 0.0f;
#pragma unroll
            for (int n = 0; n < 8; ++n) s += y[n] * y[n];
            const float f = 1.0f / sqrtf(lanes_sum<Lanes>(s) * (1.0f / RANK) + a.eps);
#pragma unroll
            for (int n = 0; n < 8; ++n) y[n] = y[n] * f * w[n];
        }
        int64_t slot, pos;
        if (!live<ROT>(a, t0 + t, slot, pos)) continue;
        const Place p = place<FMT>(a.c, slot);
        put_row<FMT>(p.row, p.scale, d, y);
    }
    // the shared keys
    const int per = a.c.rot / 8;   // 4 or 8 lanes a key
    for (uint32_t i = lane; i < left * per; i += 64) {
        const uint32_t t = i / per;
        const int e = 8 * (int)(i - t * per);
        const char *src = a.key.p + (int64_t)(t0 + t) * a.key.token_stride * E;
        const int half = a.r.rot >> 1;
        Raw<DT> raw, partner;
        raw.load(src + e * E);
        if (ROT == kHalf && e < a.r.rot) partner.load(src + (e < half ? e + half : e - half) * E);
        int64_t slot, pos;
        if (!live<ROT>(a, t0 + t, slot, pos)) continue;
        Turn<ROT> turn;
        turn.load(a.r, pos, e);
        float y[8];
        raw.get(y);
        rotate<DT, ROT>(turn, src, e, a.r, pos, partner, y);
        const Place p = place<FMT>(a.c, slot);
        put_row<FMT>(p.row, p.scale, RANK + e, y);
    }
}

template <int DT, int FMT, int ROT, int RANK>
hipError_t write_tokens(const LatentWrite &a, hipStream_t stream)
{
    // four rows a wave once that still leaves 2,048 waves or more
    const int t = a.tokens >= 4 * 2048 ? 4 : 1;
    const dim3 grid = grid_of(cdiv(a.tokens, (kThreads / 64) * t));
    if (t == 4) latent_write_kernel<DT, FMT, ROT, RANK, 4><<<grid, kThreads, 0, stream>>>(a);
    else latent_write_kernel<DT, FMT, ROT, RANK, 1><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int DT, int FMT, int ROT>
hipError_t write_rank(const LatentWrite &a, hipStream_t stream)
{
    return a.c.rank == 512 ? write_tokens<DT, FMT, ROT, 512>(a, stream)
                           : write_tokens<DT, FMT, ROT, 256>(a, stream);
}

template <int DT, int FMT>
hipError_t write_rot(const LatentWrite &a, hipStream_t stream)
{
    switch (rotation_kind(a.r)) {
    case kNoRot: return write_rank<DT, FMT, kNoRot>(a, stream);
    case kHalf: return write_rank<DT, FMT, kHalf>(a, stream);
    case kInterleaved: return write_rank<DT, FMT, kInterleaved>(a, stream);
    default: return write_rank<DT, FMT, kAnyRot>(a, stream);
    }
}

template <int DT>
hipError_t write_fmt(const LatentWrite &a, hipStream_t stream)
{
    switch (a.c.format) {
    case KVR_KV_BF16: return write_rot<DT, KVR_KV_BF16>(a, stream);
    case KVR_KV_FP16: return write_rot<DT, KVR_KV_FP16>(a, stream);
    default: return write_rot<DT, KVR_KV_FP8>(a, stream);
    }
}

// A thread has U units of eight elements, a block's width apart.
template <int FMT, int DT, int DIM, int U>
__global__ __launch_bounds__(kThreads) void latent_read_kernel(LatentRead a)
{
    constexpr int E = elem_bytes<DT>();
    constexpr int VT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // type of the values
    constexpr int Units = DIM / 8;
    const uint64_t first = (uint64_t)block_of_grid() * (kThreads * U) + threadIdx.x;
    Codes<FMT> x[U];
    bool fine[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const uint64_t i = first + j * kThreads;
        const uint32_t token = (uint32_t)(i / Units);
        fine[j] = false;
        if (i / Units >= a.tokens) continue;
        const int64_t slot = a.slots[token];
        fine[j] = slot >= 0 && slot >> a.c.page_shift < a.c.n_pages;
        if (!fine[j]) {
            if (slot >= 0 && a.status) *a.status = KVR_E_DOMAIN;
            continue;
        }
        const Place p = place<FMT>(a.c, slot);
        x[j].load(p.row, p.scale, 8 * (int)(i - (uint64_t)token * Units));
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const uint64_t i = first + j * kThreads;
        const uint32_t token = (uint32_t)(i / Units);
        if (i / Units >= a.tokens) return;
        uint32_t p[4] = {0, 0, 0, 0};
        if (fine[j]) x[j].get(p);
        char *dst = a.out.p + ((int64_t)token * a.out.token_stride + 8 * (int)(i - (uint64_t)token * Units)) * E;
        if (DT == VT) {
            store16<false>(reinterpret_cast<u32x4 *>(dst), u32x4{p[0], p[1], p[2], p[3]});
            continue;
        }
        float y[8];
#pragma unroll
        for (int n = 0; n < 4; ++n) unpack16<VT>(p[n], y[2 * n], y[2 * n + 1]);
        store8<DT>(dst, y);
    }
}

template <int FMT, int DT, int DIM>
hipError_t read_units(const LatentRead &a, hipStream_t stream)
{
    const int64_t units = (int64_t)a.tokens * (DIM / 8);
    // four units a thread once that still leaves 2,048 waves or more
    const bool large = units >= 4 * 2048 * 64;
    const dim3 grid = grid_of(cdiv(units, kThreads * (large ? 4 : 1)));
    if (!large) latent_read_kernel<FMT, DT, DIM, 1><<<grid, kThreads, 0, stream>>>(a);
    else latent_read_kernel<FMT, DT, DIM, 4><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int FMT, int DT>
hipError_t read_dim(const LatentRead &a, hipStream_t stream)
{
    switch (a.c.rank + a.c.rot) {
    case 288: return read_units<FMT, DT, 288>(a, stream);
    case 320: return read_units<FMT, DT, 320>(a, stream);
    case 544: return read_units<FMT, DT, 544>(a, stream);
    default: return read_units<FMT, DT, 576>(a, stream);
    }
}

template <int FMT>
hipError_t read_out(const LatentRead &a, hipStream_t stream)
{
    switch (a.out.dtype) {
    case KVR_DT_BF16: return read_dim<FMT, KVR_DT_BF16>(a, stream);
    case KVR_DT_FP16: return read_dim<FMT, KVR_DT_FP16>(a, stream);
    default: return read_dim<FMT, KVR_DT_FP32>(a, stream);
    }
}

}  // namespace

hipError_t launch_latent_write(const LatentWrite &a, hipStream_t stream)
{
    switch (a.latent.dtype) {
    case KVR_DT_BF16: return write_fmt<KVR_DT_BF16>(a, stream);
    case KVR_DT_FP16: return write_fmt<KVR_DT_FP16>(a, stream);
    default: return write_fmt<KVR_DT_FP32>(a, stream);
    }
}

hipError_t launch_latent_read(const LatentRead &a, hipStream_t stream)
{
    switch (a.c.format) {
    case KVR_KV_BF16: return read_out<KVR_KV_BF16>(a, stream);
    case KVR_KV_FP16: return read_out<KVR_KV_FP16>(a, stream);
    default: return read_out<KVR_KV_FP8>(a, stream);
    }
}

}  // namespace kv
}  // namespace kvr
