// Attention over a bfloat16 latent cache.
#include "kvr_latent_attention.h"

namespace kvr {
namespace kv {

hipError_t launch_latent_bf16(const LatentAttention &l, dim3 grid, hipStream_t stream)
{
    return launch_latent_format<KVR_KV_BF16>(l, grid, stream);
}

}  // namespace kv
}  // namespace kvr
