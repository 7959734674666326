// Attention over the latent cache: the launch plan.
#include <algorithm>
#include <cmath>

#include "kvr_latent.h"

namespace kvr {
namespace kv {

size_t plan_latent_attention(LatentAttention &l)
{
    Attention &a = l.a;
    const int64_t rows = (int64_t)a.max_q * a.group;
    const int64_t longest = cdiv(a.max_kv, kStep);
    const int share = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;   // tiles of 16 rows a block
    a.block_rows = 16 * share;
    a.min_steps = 8;
    // Blocks that are resident at once, by LDS.  Sequences are cut into whole numbers of parts, to
    // the nearest, so that n of them come to about sqrt(n) / 3 parts more or less than planned,
    // and one more than there is room for would begin another round.
    const int64_t blocks = std::min<int64_t>((int64_t)a.n_seqs * cdiv(rows, a.block_rows),
                                             a.n_queries * a.group / a.block_rows + a.n_seqs);
    const int64_t slots = 256;
    a.target = (int32_t)(slots - (int64_t)std::sqrt((double)std::min(blocks, slots)));
    a.max_items = (int32_t)std::max<int64_t>(
        1, std::min(a.target + blocks, blocks * cdiv(longest, a.min_steps)));
    a.direct = 0;
    if (longest <= a.min_steps) {
        const int64_t room = cdiv(rows, a.block_rows);
        if (a.max_pages > 0 && (room == 1 || a.n_seqs * room <= 1024)) {
            a.direct = (int32_t)room;
            a.max_items = (int32_t)std::max<int64_t>(1, a.n_seqs * room);
        }
        return 0;
    }
    return (size_t)a.max_items * a.block_rows * (l.c.rank + 4) * sizeof(float);
}

hipError_t launch_latent_attention(const LatentAttention &l, hipStream_t stream)
{
    const dim3 grid((unsigned)l.a.max_items);
    hipError_t e;
    switch (l.c.format) {
    case KVR_KV_BF16: e = launch_latent_bf16(l, grid, stream); break;
    case KVR_KV_FP16: e = launch_latent_fp16(l, grid, stream); break;
    default: e = launch_latent_fp8(l, grid, stream);
    }
    if (e != hipSuccess || l.a.part_o == nullptr) return e;
    return launch_join(l.a, stream);
}

}  // namespace kv
}  // namespace kvr
