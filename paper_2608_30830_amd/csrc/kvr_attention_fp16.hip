// Attention over a half-precision cache.
#include "kvr_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_attention_fp16(const Attention &a, dim3 grid, hipStream_t stream)
{
    return launch_dim<KVR_KV_FP16, KVR_DT_FP16>(a, grid, stream);
}

}  // namespace kv
}  // namespace kvr
