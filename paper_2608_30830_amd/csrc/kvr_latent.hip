// Attention over the latent cache: the launch plan.
#include <algorithm>

#include "kvr_latent.h"

namespace kvr {
namespace kv {

constexpr int kSlots = 256;   // blocks that are resident at once: one on each CU, by LDS

size_t plan_latent_attention(LatentAttention &l)
{
    Attention &a = l.a;
    const int64_t rows = (int64_t)a.max_q * a.group;
    const int64_t longest = cdiv(a.max_kv, kStep);
    // Registers hold 64 rows of 512 elements a block, or 128 of 256 (64 sequences of 16,384 tokens,
    // 128 heads: 229 us in blocks of 128 rows, 334 in blocks of 64); the rows of a sequence are divided
    // evenly among as few blocks as that allows, in tiles of 16.
    const int64_t most = rows <= 64 || l.c.rank == 512 ? 64 : 128;
    a.block_rows = rows <= 16 ? 16 : (int32_t)(16 * cdiv(rows, 16 * cdiv(rows, most)));
    // (one sequence of 1,000 tokens: 17.3 us in parts of four steps, 19.7 of eight; with more rows a
    // part's way through memory costs as much as about eight steps)
    a.min_steps = rows <= 16 ? 4 : 8;
    l.span = (int32_t)std::min<int64_t>(cdiv(rows, a.block_rows), 32);   // an XCD has 32 CUs
    const int64_t blocks = std::min<int64_t>((int64_t)a.n_seqs * cdiv(rows, a.block_rows),
                                             a.n_queries * a.group / a.block_rows + a.n_seqs);
    a.target = kSlots;
    a.fit = kSlots;   // a block more than there is room for begins another round
    // (fitted_steps cuts for several rounds only where the row blocks exceed half a round)
    a.max_items = (int32_t)std::max<int64_t>(
        1, std::min(2 * blocks > kSlots ? blocks + 2 * kSlots : kSlots, blocks * cdiv(longest, a.min_steps)));
    a.direct = 0;
    if (longest <= a.min_steps) {
        const int64_t room = cdiv(rows, a.block_rows);
        if (a.max_pages > 0 && (room == 1 || a.n_seqs * room <= 1024)) {
            a.direct = (int32_t)room;
            a.max_items = (int32_t)std::max<int64_t>(1, a.n_seqs * room);
        }
        return 0;
    }
    // and a word for the steps of a part
    return (size_t)a.max_items * a.block_rows * (l.c.rank + 4) * sizeof(float) + 16;
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
