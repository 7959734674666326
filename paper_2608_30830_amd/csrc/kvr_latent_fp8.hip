// Attention over a 8-bit latent cache.
#include "kvr_latent_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_latent_fp8(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    return launch_latent_format<KVR_KV_FP8>(l, grid, stream);
}

}  // namespace kv
}  // namespace kvr
