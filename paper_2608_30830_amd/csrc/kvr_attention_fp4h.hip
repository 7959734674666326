// Attention over an e2m1 cache, half-precision queries.
#include "kvr_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_attention_fp4h(const Attention &a, dim3 grid, hipStream_t stream)
{
    return launch_dim<KVR_KV_FP4, KVR_DT_FP16>(a, grid, stream);
}

}  // namespace kv
}  // namespace kvr
