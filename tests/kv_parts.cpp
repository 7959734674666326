// The items of attention calls as the host plans them and the device counts them, without
// a GPU.  Reads calls from standard input: q_heads kv_heads max_q max_kv n_queries n_seqs, then n_seqs
// + 1 first queries and n_seqs lengths; prints for each what a call's sequences come to.
#include <cstdio>
#include <vector>

#include "kvr_parts.h"

int main()
{
    using namespace kvr::kv;
    int q_heads, kv_heads, max_q, max_kv, n_seqs;
    long long n_queries;
    while (std::scanf("%d %d %d %d %lld %d", &q_heads, &kv_heads, &max_q, &max_kv, &n_queries,
                      &n_seqs) == 6) {
        std::vector<int32_t> cu(n_seqs + 1), len(n_seqs);
        for (int32_t &x : cu)
            if (std::scanf("%d", &x) != 1) return 1;
        for (int32_t &x : len)
            if (std::scanf("%d", &x) != 1) return 1;
        Attention a{};
        int status = 0;
        a.c.n_heads = kv_heads, a.c.dim = 128, a.c.page_shift = 4;
        a.q_heads = q_heads, a.group = q_heads / kv_heads;
        a.max_q = max_q, a.max_kv = max_kv, a.n_queries = n_queries, a.n_seqs = n_seqs;
        a.max_pages = (max_kv + 15) / 16;
        a.cu_q = cu.data(), a.kv_len = len.data(), a.status = &status;
        const size_t bytes = plan_attention(a);
        const int64_t room = (int64_t)(bytes / sizeof(float) / (a.c.dim + 4)) / kv_heads / a.block_rows;
        std::vector<int> steps(n_seqs), rbs(n_seqs);
        int64_t total = 0;
        for (int b = 0; b < n_seqs; ++b) {
            int l, nq, q0;
            sequence(a, b, l, nq, q0);
            steps[b] = steps_of(l, nq), rbs[b] = row_blocks_of(a, nq);
            total += (int64_t)steps[b] * rbs[b];
        }
        const int per = part_size(a, total);
        int64_t base = 0, used = 0, left = 0, whole = 0;   // items; of joined sequences; sequences left out
        for (int b = 0; b < n_seqs; ++b) {
            const int parts = parts_of(steps[b], per);
            const int64_t end = base + (int64_t)parts * rbs[b];
            if (parts > 1) {
                if (planned(a, base, parts, rbs[b])) used = end > used ? end : used, ++whole;
                else ++left;
            }
            base = end;
        }
        std::printf("%d %lld %lld %d %lld %lld %lld %lld\n", status, (long long)a.max_items,
                    (long long)room, per, (long long)base, (long long)used, (long long)whole,
                    (long long)left);
    }
    return 0;
}
