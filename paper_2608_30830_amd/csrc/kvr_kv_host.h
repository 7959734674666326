// Checks of arguments that the entry points of the caches share.
#pragma once

#include <cstdint>

#include "kvr.h"
#include "kvr_kv.h"

namespace {

using kvr::kv::Rotary;
using kvr::kv::Rows;

constexpr int64_t kMaxRows = INT32_MAX;

inline bool dtype_ok(int32_t t) { return t == KVR_DT_BF16 || t == KVR_DT_FP16 || t == KVR_DT_FP32; }
inline int64_t dtype_bytes(int32_t t) { return t == KVR_DT_FP32 ? 4 : 2; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The strides of a single token or head do not matter.
inline Rows rows(const void *p, int64_t tokens, int64_t token_stride, int64_t heads, int64_t head_stride,
          int32_t dtype)
{
    return Rows{static_cast<char *>(const_cast<void *>(p)), tokens > 1 ? token_stride : 0,
                heads > 1 ? head_stride : 0, dtype};
}

inline bool rows_aligned(const Rows &r)
{
    const int64_t e = dtype_bytes(r.dtype);
    return aligned16(r.p) && r.token_stride >= 0 && r.head_stride >= 0 &&
           r.token_stride * e % 16 == 0 && r.head_stride * e % 16 == 0;
}

inline int check_rotary(const int32_t *d_pos, const float *d_table, int64_t n_pos, int32_t rot,
                 int32_t head_dim, int32_t flags, Rotary &out)
{
    if (!d_pos) return KVR_E_NULL;
    if (rot < 2 || rot % 2 != 0 || rot > head_dim || rot > 2 * kvr::kv::kMaxFreq || n_pos < 1)
        return KVR_E_SIZE;
    if (reinterpret_cast<uintptr_t>(d_table) & 3) return KVR_E_LAYOUT;
    if (flags & ~(KVR_ROTARY_INTERLEAVED | KVR_ROTARY_ADJOINT)) return KVR_E_METHOD;
    out.t = d_table;
    out.pos = d_pos;
    out.n_pos = n_pos;
    out.rot = rot;
    out.interleaved = (flags & KVR_ROTARY_INTERLEAVED) != 0;
    out.sign = (flags & KVR_ROTARY_ADJOINT) ? -1.0f : 1.0f;
    return KVR_OK;
}

#define KVR_TRY(expr)                                \
    do {                                             \
        if ((expr) != hipSuccess) return KVR_E_HIP;  \
    } while (0)

}  // namespace
