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
// permutes), dim / 8 lanes a row; and in large calls four heads of its token, so
// that their loads are in flight together and the token's slot and table row are
// read once for them.  8 heads of 128: 131,072 tokens read from 8 bits in 141 us
// (5.8 TB/s), 32,749 written in 4 bits in 34 us (5.0 TB/s) and read in 27 (6.2).
#include "kvr_rows.h"

namespace kvr {
namespace kv {
namespace {

constexpr int kThreads = 256;

struct WriteArgs {
    Cache c;
    Rows k, v;
    Rotary r;
    const int64_t *slots;
    uint32_t groups;       // tokens * head_groups
    int32_t head_groups;   // a lane has the heads hg, hg + head_groups, ...
    int32_t lane_shift;    // log2 of the lanes of a row
    int *status;
};

template <int DT, int FMT, int ROT, int HPT>
__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a)
{
    constexpr int E = elem_bytes<DT>();
    const uint32_t i = block_of_grid() * (uint32_t)(kThreads >> a.lane_shift) +
                       (threadIdx.x >> a.lane_shift);
    const int d = 8 * (threadIdx.x & ((1 << a.lane_shift) - 1));
    if (i >= a.groups || d >= a.c.dim) return;   // whole quads: dim is a multiple of 32
    const uint32_t token = i / (uint32_t)a.head_groups;
    const int hg = (int)(i - token * (uint32_t)a.head_groups);
    const bool key = blockIdx.y == 0;
    const Rows &in = key ? a.k : a.v;
    const char *src = in.p + (int64_t)token * in.token_stride * E;
    const int64_t slot = a.slots[token];
    const int64_t pos = ROT != kNoRot ? a.r.pos[token] : 0;
    Raw<DT> x[HPT], y[HPT];
    const int half = a.r.rot >> 1;
    const bool pair = ROT == kHalf && key && d < a.r.rot;
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        const int h = hg + j * a.head_groups;
        if (h < a.c.n_heads) {
            const char *row = src + (int64_t)h * in.head_stride * E;
            x[j].load(row + d * E);
            if (pair) y[j].load(row + (d < half ? d + half : d - half) * E);
        }
    }
    if (slot < 0) return;
    const int64_t page = slot >> a.c.page_shift;
    if (page >= a.c.n_pages || (ROT != kNoRot && (pos < 0 || pos >= a.r.n_pos))) {
        if (a.status) *a.status = KVR_E_DOMAIN;
        return;
    }
    Turn<ROT> turn;
    turn.on = false;
    if (key) turn.load(a.r, pos, d);
    const int64_t off = slot & ((1ll << a.c.page_shift) - 1);
    char *dst = (key ? a.c.k : a.c.v) + page * a.c.page_stride + off * a.c.token_stride;
    uint8_t *sc = nullptr;
    if (FMT == KVR_KV_FP8 || FMT == KVR_KV_FP4)
        sc = (key ? a.c.ks : a.c.vs) + page * a.c.spage_stride + off * a.c.stoken_stride;
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        const int h = hg + j * a.head_groups;
        if (h >= a.c.n_heads) break;
        float z[8];
        x[j].get(z);
        if (key) rotate<DT, ROT>(turn, src + (int64_t)h * in.head_stride * E, d, a.r, pos, y[j], z);
        put_row<FMT>(dst + h * a.c.head_stride, sc + h * a.c.shead_stride, d, z);
    }
}

struct ReadArgs {
    Cache c;
    Rows k, v;
    const int64_t *slots;
    uint32_t groups;
    int32_t head_groups, lane_shift;
    int *status;
};

template <int FMT, int DT, int HPT, bool Stream = false>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a)
{
    constexpr int E = elem_bytes<DT>();
    constexpr int VT = FMT == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16;   // type of the values
    const uint32_t i = block_of_grid() * (uint32_t)(kThreads >> a.lane_shift) +
                       (threadIdx.x >> a.lane_shift);
    const int d = 8 * (threadIdx.x & ((1 << a.lane_shift) - 1));
    if (i >= a.groups || d >= a.c.dim) return;
    const uint32_t token = i / (uint32_t)a.head_groups;
    const int hg = (int)(i - token * (uint32_t)a.head_groups);
    const bool key = blockIdx.y == 0;
    const Rows &out = key ? a.k : a.v;
    char *dst = out.p + ((int64_t)token * out.token_stride + d) * E;
    const int64_t slot = a.slots[token];
    const int64_t page = slot >> a.c.page_shift;
    const bool live = slot >= 0 && page < a.c.n_pages;
    if (!live && slot >= 0 && a.status) *a.status = KVR_E_DOMAIN;
    const int64_t off = slot & ((1ll << a.c.page_shift) - 1);
    const char *src = (key ? a.c.k : a.c.v) + page * a.c.page_stride + off * a.c.token_stride;
    const uint8_t *sc = nullptr;
    if (Codes<FMT>::Quant)
        sc = (key ? a.c.ks : a.c.vs) + page * a.c.spage_stride + off * a.c.stoken_stride;
    Codes<FMT> x[HPT];
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        const int h = hg + j * a.head_groups;
        if (live && h < a.c.n_heads)
            x[j].load(src + h * a.c.head_stride, sc + h * a.c.shead_stride, d);
    }
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        const int h = hg + j * a.head_groups;
        if (h >= a.c.n_heads) break;
        uint32_t p[4] = {0, 0, 0, 0};
        if (live) x[j].get(p);
        char *row = dst + (int64_t)h * out.head_stride * E;
        if (DT == VT) {
            store16<Stream>(reinterpret_cast<u32x4 *>(row), u32x4{p[0], p[1], p[2], p[3]});
            continue;
        }
        float y[8];
#pragma unroll
        for (int n = 0; n < 4; ++n) unpack16<VT>(p[n], y[2 * n], y[2 * n + 1]);
        store8<DT, Stream>(row, y);
    }
}

int lane_shift(int dim)
{
    int s = 2;
    while ((8 << s) < dim) ++s;
    return s;
}

// Heads of a lane: four once that leaves 2,048 waves or more of each of k and v.
int heads_per_lane(int64_t tokens, const Cache &c)
{
    return c.n_heads >= 4 && tokens * c.n_heads * c.dim / 8 >= 4 * 2048 * 64 ? 4 : 1;
}
template <class Args>
dim3 plan(Args &a, int64_t tokens, int hpt)
{
    a.head_groups = (a.c.n_heads + hpt - 1) / hpt;
    a.groups = (uint32_t)(tokens * a.head_groups);
    a.lane_shift = lane_shift(a.c.dim);
    return grid_of(cdiv(a.groups, kThreads >> a.lane_shift), 2);
}

template <int DT, int FMT, int ROT>
hipError_t write_heads(WriteArgs &a, int64_t tokens, hipStream_t stream)
{
    const int hpt = heads_per_lane(tokens, a.c);
    const dim3 grid = plan(a, tokens, hpt);
    if (hpt == 4) write_kernel<DT, FMT, ROT, 4><<<grid, kThreads, 0, stream>>>(a);
    else write_kernel<DT, FMT, ROT, 1><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int DT, int FMT>
hipError_t write_rot(WriteArgs &a, int64_t tokens, hipStream_t stream)
{
    switch (rotation_kind(a.r)) {
    case kNoRot: return write_heads<DT, FMT, kNoRot>(a, tokens, stream);
    case kHalf: return write_heads<DT, FMT, kHalf>(a, tokens, stream);
    case kInterleaved: return write_heads<DT, FMT, kInterleaved>(a, tokens, stream);
    default: return write_heads<DT, FMT, kAnyRot>(a, tokens, stream);
    }
}

template <int DT>
hipError_t write_fmt(WriteArgs &a, int64_t tokens, hipStream_t stream)
{
    switch (a.c.format) {
    case KVR_KV_BF16: return write_rot<DT, KVR_KV_BF16>(a, tokens, stream);
    case KVR_KV_FP16: return write_rot<DT, KVR_KV_FP16>(a, tokens, stream);
    case KVR_KV_FP8: return write_rot<DT, KVR_KV_FP8>(a, tokens, stream);
    default: return write_rot<DT, KVR_KV_FP4>(a, tokens, stream);
    }
}

template <int FMT, int DT>
hipError_t read_heads(ReadArgs &a, int64_t tokens, hipStream_t stream)
{
    const int hpt = heads_per_lane(tokens, a.c);
    const dim3 grid = plan(a, tokens, hpt);
    const bool large = hpt == 4 && streams(2 * tokens * a.c.n_heads * a.c.dim, a.c.dim, DT);
    if (large) read_kernel<FMT, DT, 4, DT != KVR_DT_FP32><<<grid, kThreads, 0, stream>>>(a);
    else if (hpt == 4) read_kernel<FMT, DT, 4><<<grid, kThreads, 0, stream>>>(a);
    else read_kernel<FMT, DT, 1><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int FMT>
hipError_t read_out(ReadArgs &a, int64_t tokens, hipStream_t stream)
{
    switch (a.k.dtype) {
    case KVR_DT_BF16: return read_heads<FMT, KVR_DT_BF16>(a, tokens, stream);
    case KVR_DT_FP16: return read_heads<FMT, KVR_DT_FP16>(a, tokens, stream);
    default: return read_heads<FMT, KVR_DT_FP32>(a, tokens, stream);
    }
}

}  // namespace

hipError_t launch_cache_write(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                              const int64_t *slots, const Rotary &r, int *status,
                              hipStream_t stream)
{
    WriteArgs a{};
    a.c = c, a.k = k, a.v = v, a.r = r, a.slots = slots, a.status = status;
    switch (k.dtype) {
    case KVR_DT_BF16: return write_fmt<KVR_DT_BF16>(a, tokens, stream);
    case KVR_DT_FP16: return write_fmt<KVR_DT_FP16>(a, tokens, stream);
    default: return write_fmt<KVR_DT_FP32>(a, tokens, stream);
    }
}

hipError_t launch_cache_read(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                             const int64_t *slots, int *status, hipStream_t stream)
{
    ReadArgs a{};
    a.c = c, a.k = k, a.v = v, a.slots = slots, a.status = status;
    switch (c.format) {
    case KVR_KV_BF16: return read_out<KVR_KV_BF16>(a, tokens, stream);
    case KVR_KV_FP16: return read_out<KVR_KV_FP16>(a, tokens, stream);
    case KVR_KV_FP8: return read_out<KVR_KV_FP8>(a, tokens, stream);
    default: return read_out<KVR_KV_FP4>(a, tokens, stream);
    }
}

}  // namespace kv
}  // namespace kvr
