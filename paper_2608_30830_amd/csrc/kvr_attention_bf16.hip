// Attention over a bfloat16 cache.
#include "kvr_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_attention_bf16(const Attention &a, dim3 grid, hipStream_t stream)
{
    return launch_dim<KVR_KV_BF16, KVR_DT_BF16>(a, grid, stream);
}

}  // namespace kv
}  // namespace kvr
