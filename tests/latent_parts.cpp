// The parts of latent attention calls as the host plans them and the device counts them, without
// a GPU.  Reads calls from standard input: n_heads rank max_q max_kv n_seqs, then n_seqs new tokens and
// n_seqs lengths; prints what a call's sequences come to.
#include <cstdio>
#include <vector>

#include "kvr_latent.h"
#include "kvr_parts.h"

int main()
{
    using namespace kvr::kv;
    int heads, rank, max_q, max_kv, n_seqs;
    while (std::scanf("%d %d %d %d %d", &heads, &rank, &max_q, &max_kv, &n_seqs) == 5) {
        std::vector<int32_t> nq(n_seqs), len(n_seqs);
        LatentAttention l{};
        Attention &a = l.a;
        for (int32_t &x : nq) {
            if (std::scanf("%d", &x) != 1) return 1;
            a.n_queries += x;
        }
        for (int32_t &x : len)
            if (std::scanf("%d", &x) != 1) return 1;
        l.c.rank = a.c.dim = rank;
        a.c.n_heads = 1, a.c.page_shift = 4;
        a.q_heads = a.group = heads;
        a.max_q = max_q, a.max_kv = max_kv, a.n_seqs = n_seqs;
        a.max_pages = (max_kv + 15) / 16;
        const size_t bytes = plan_latent_attention(l);
        int64_t total = 0, blocks = 0, most = 0;
        int calls = 0;
        for (int b = 0; b < n_seqs; ++b) {
            const int s = steps_of(len[b], nq[b]), rb = row_blocks_of(a, nq[b]);
            total += (int64_t)s * rb;
            blocks += s > 0 ? rb : 0;
            most = s > most ? s : most;
        }
        auto count = [&](int per) {
            int64_t n = 0;
            for (int b = 0; b < n_seqs; ++b)
                n += (int64_t)fitted_parts(steps_of(len[b], nq[b]), per) * row_blocks_of(a, nq[b]);
            ++calls;
            return n;
        };
        const int per = fitted_steps(a, total, blocks, count);
        std::printf("%d %lld %lld %d %lld %lld %lld %lld %d %d\n", a.direct, (long long)a.max_items,
                    (long long)(bytes / sizeof(float) / (rank + 4) / a.block_rows), per, (long long)count(per),
                    (long long)total, (long long)blocks, (long long)most, a.fit, calls - 1);
    }
    return 0;
}
