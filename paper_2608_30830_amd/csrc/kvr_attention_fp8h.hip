// Attention over an e4m3 cache, half-precision queries.
#include "kvr_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_attention_fp8h(const Attention &a, dim3 grid, hipStream_t stream)
{
    return launch_dim<KVR_KV_FP8, KVR_DT_FP16>(a, grid, stream);
}

}  // namespace kv
}  // namespace kvr
