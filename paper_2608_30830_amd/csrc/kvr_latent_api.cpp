// C ABI of the latent cache: validation on the host, launches.
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "kvr.h"
#include "kvr_kv_host.h"
#include "kvr_latent.h"

namespace {

using kvr::kv::LatentAttention;
using kvr::kv::LatentRead;
using kvr::kv::Latents;
using kvr::kv::LatentWrite;
using kvr::kv::Prompt;

int check_latents(const kvr_latent_cache *c, Latents &out)
{
    if (!c) return KVR_E_NULL;
    if (c->format < KVR_KV_BF16 || c->format > KVR_KV_FP8) return KVR_E_LAYOUT;
    const bool quant = c->format == KVR_KV_FP8;
    if (!c->data || (quant && !c->scale)) return KVR_E_NULL;
    if (c->n_pages < 1 || c->n_pages > INT32_MAX) return KVR_E_SIZE;
    const int32_t ps = c->page_size;
    if (ps < 16 || ps > 32768 || (ps & (ps - 1)) != 0) return KVR_E_LAYOUT;
    if ((c->rank != 256 && c->rank != 512) || (c->rot != 32 && c->rot != 64)) return KVR_E_LAYOUT;
    if (!aligned16(c->data)) return KVR_E_LAYOUT;
    // the stride of a single page does not matter
    const int64_t page = c->n_pages > 1 ? c->page_stride : 0;
    const int64_t spage = c->n_pages > 1 ? c->scale_page_stride : 0;
    if (page < 0 || page % 16 != 0 || c->token_stride < 0 || c->token_stride % 16 != 0 ||
        c->token_stride > (1 << 26))
        return KVR_E_LAYOUT;
    if (quant && (spage < 0 || c->scale_token_stride < 0 || c->scale_token_stride > (1 << 26)))
        return KVR_E_LAYOUT;
    out.rows = static_cast<char *>(c->data);
    out.scale = static_cast<uint8_t *>(c->scale);
    out.page_stride = page;
    out.token_stride = c->token_stride;
    out.spage_stride = spage;
    out.stoken_stride = c->scale_token_stride;
    out.n_pages = c->n_pages;
    out.page_shift = __builtin_ctz((unsigned)ps);
    out.rank = c->rank;
    out.rot = c->rot;
    out.format = c->format;
    return KVR_OK;
}

// |scale| * log2(e), and not zero: that keeps -infinity times it -infinity.
float scale_log2(float scale)
{
    const float s = (float)(std::fabs((double)scale) * 1.4426950408889634);
    return s == 0.0f ? FLT_MIN : s;
}

}  // namespace

extern "C" {

int kvr_latent_write(const kvr_latent_cache *cache, const void *d_latent, const void *d_key,
                     int32_t dtype, int64_t n_tokens, int64_t latent_stride, int64_t key_stride,
                     const void *d_norm, float eps, const int64_t *d_slots, const int32_t *d_pos,
                     const float *d_table, int64_t n_pos, int32_t rot_dim, int32_t flags,
                     int32_t *d_status, void *hip_stream)
{
    LatentWrite a{};
    int rc = check_latents(cache, a.c);
    if (rc != KVR_OK) return rc;
    if (n_tokens < 0 || n_tokens > kMaxRows) return KVR_E_SIZE;
    if (!dtype_ok(dtype)) return KVR_E_LAYOUT;
    if (d_norm && (!std::isfinite(eps) || eps < 0.0f)) return KVR_E_GRID;
    if (n_tokens == 0) return KVR_OK;
    if (!d_latent || !d_key || !d_slots) return KVR_E_NULL;
    if (d_table) {
        rc = check_rotary(d_pos, d_table, n_pos, rot_dim, a.c.rot, flags, a.r);
        if (rc != KVR_OK) return rc;
    }
    a.latent = rows(d_latent, n_tokens, latent_stride, 1, 0, dtype);
    a.key = rows(d_key, n_tokens, key_stride, 1, 0, dtype);
    if (!rows_aligned(a.latent) || !rows_aligned(a.key) || !aligned16(d_norm)) return KVR_E_LAYOUT;
    a.norm = static_cast<const char *>(d_norm);
    a.eps = eps;
    a.slots = d_slots;
    a.tokens = (uint32_t)n_tokens;
    a.status = d_status;
    KVR_TRY(kvr::kv::launch_latent_write(a, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_latent_read(const kvr_latent_cache *cache, const int64_t *d_slots, int64_t n_tokens,
                    void *d_out, int32_t dtype, int64_t out_stride, int32_t *d_status,
                    void *hip_stream)
{
    LatentRead a{};
    const int rc = check_latents(cache, a.c);
    if (rc != KVR_OK) return rc;
    if (n_tokens < 0 || n_tokens > kMaxRows) return KVR_E_SIZE;
    if (!dtype_ok(dtype)) return KVR_E_LAYOUT;
    if (n_tokens == 0) return KVR_OK;
    if (!d_out || !d_slots) return KVR_E_NULL;
    a.out = rows(d_out, n_tokens, out_stride, 1, 0, dtype);
    if (!rows_aligned(a.out)) return KVR_E_LAYOUT;
    a.slots = d_slots;
    a.tokens = (uint32_t)n_tokens;
    a.status = d_status;
    KVR_TRY(kvr::kv::launch_latent_read(a, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_latent_attention(const kvr_latent_cache *cache, const kvr_sequences *seqs, const void *d_q,
                         int32_t dtype, int32_t n_heads, int64_t q_token_stride,
                         int64_t q_head_stride, const uint64_t *d_tree_mask, int32_t mask_words,
                         float scale, void *d_out, int64_t out_token_stride,
                         int64_t out_head_stride, float *d_lse, int32_t *d_status, void *d_ws,
                         size_t *ws_bytes, void *hip_stream)
{
    LatentAttention l{};
    kvr::kv::Attention &a = l.a;
    const int rc = check_latents(cache, l.c);
    if (rc != KVR_OK) return rc;
    if (!seqs || !ws_bytes) return KVR_E_NULL;
    if (dtype != (l.c.format == KVR_KV_FP16 ? KVR_DT_FP16 : KVR_DT_BF16)) return KVR_E_LAYOUT;
    if (n_heads < 1 || seqs->n_seqs < 0 || seqs->n_seqs > kvr::kv::kMaxSeqs || seqs->max_q < 1 ||
        seqs->max_kv < 1 || seqs->max_kv > (1 << 30) || seqs->n_queries < 0 ||
        seqs->n_queries > INT32_MAX || seqs->max_pages < 0 || seqs->pages_stride < 0 ||
        (int64_t)seqs->max_q * n_heads > (1 << 24))
        return KVR_E_SIZE;
    if (d_tree_mask && (mask_words < 1 || (int64_t)mask_words * 64 < seqs->max_q)) return KVR_E_SIZE;
    if (!std::isfinite(scale)) return KVR_E_GRID;
    a.c.n_pages = l.c.n_pages;
    a.c.page_shift = l.c.page_shift;
    a.c.n_heads = 1;
    a.c.dim = l.c.rank;
    a.c.format = l.c.format;
    a.group = n_heads;
    a.q_heads = n_heads;
    a.n_seqs = seqs->n_seqs;
    a.max_q = seqs->max_q;
    a.max_kv = seqs->max_kv;
    a.n_queries = seqs->n_queries;
    a.max_pages = seqs->max_pages;
    const size_t need = kvr::kv::plan_latent_attention(l);
    if (!d_ws) {
        *ws_bytes = need;
        return KVR_OK;
    }
    if ((reinterpret_cast<uintptr_t>(d_ws) & 255) != 0 || *ws_bytes < need) return KVR_E_WORKSPACE;
    if (seqs->n_seqs == 0 || seqs->n_queries == 0) return KVR_OK;
    if (!d_q || !d_out || !seqs->d_cu_q || !seqs->d_kv_len || !seqs->d_pages) return KVR_E_NULL;
    a.q = rows(d_q, a.n_queries, q_token_stride, n_heads, q_head_stride, dtype);
    a.out = rows(d_out, a.n_queries, out_token_stride, n_heads, out_head_stride, dtype);
    if (!rows_aligned(a.q) || !rows_aligned(a.out)) return KVR_E_LAYOUT;
    a.lse = d_lse;
    a.cu_q = seqs->d_cu_q;
    a.kv_len = seqs->d_kv_len;
    a.pages = seqs->d_pages;
    a.pages_stride = seqs->pages_stride;
    a.mask = d_tree_mask;
    a.words = mask_words;
    a.scale2 = scale_log2(scale);
    a.negate = scale < 0.0f;
    a.status = d_status;
    if (need) {
        const size_t cells = need / sizeof(float) / (size_t)(l.c.rank + 4);
        a.part_o = static_cast<float *>(d_ws);
        a.part_ml = reinterpret_cast<float4 *>(a.part_o + cells * (size_t)l.c.rank);
        a.chosen = reinterpret_cast<int32_t *>(a.part_ml + cells);
    }
    KVR_TRY(kvr::kv::launch_latent_attention(l, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_latent_prompt(const kvr_prompt *prompt, const void *d_q, int32_t dtype,
                      int64_t q_token_stride, int64_t q_head_stride, const void *d_k,
                      int64_t k_token_stride, int64_t k_head_stride, const void *d_k_rot,
                      int64_t k_rot_stride, const void *d_v, int64_t v_token_stride,
                      int64_t v_head_stride, float scale, void *d_out, int64_t out_token_stride,
                      int64_t out_head_stride, float *d_lse, int32_t *d_status, void *d_ws,
                      size_t *ws_bytes, void *hip_stream)
{
    if (!prompt || !ws_bytes) return KVR_E_NULL;
    const kvr_prompt &c = *prompt;
    if (dtype != KVR_DT_BF16 && dtype != KVR_DT_FP16) return KVR_E_LAYOUT;
    if ((c.nope != 64 && c.nope != 128) || (c.rot != 32 && c.rot != 64)) return KVR_E_LAYOUT;
    if (c.causal != 0 && c.causal != 1) return KVR_E_METHOD;
    if (c.n_seqs < 0 || c.n_seqs > kvr::kv::kMaxSeqs || c.max_q < 1 || c.max_k < 1 ||
        c.max_k > (1 << 30) || c.n_queries < 0 || c.n_queries > INT32_MAX || c.n_keys < 0 ||
        c.n_keys > INT32_MAX || c.n_kv_heads < 1 || c.n_kv_heads > 1024 || c.n_q_heads < c.n_kv_heads ||
        c.n_q_heads > 4096 || c.n_q_heads % c.n_kv_heads != 0 ||
        (int64_t)c.max_q * c.n_q_heads > (1 << 30) ||
        c.n_queries > (int64_t(1) << 36) / c.n_q_heads)
        return KVR_E_SIZE;
    if (!std::isfinite(scale)) return KVR_E_GRID;
    Prompt p{};
    p.n_queries = c.n_queries;
    p.n_keys = c.n_keys;
    p.n_seqs = c.n_seqs;
    p.max_q = c.max_q;
    p.max_k = c.max_k;
    p.q_heads = c.n_q_heads;
    p.kv_heads = c.n_kv_heads;
    p.group = c.n_q_heads / c.n_kv_heads;
    p.nope = c.nope;
    p.rot = c.rot;
    p.causal = c.causal;
    const size_t need = kvr::kv::plan_prompt(p);
    if (!d_ws) {
        *ws_bytes = need;
        return KVR_OK;
    }
    if ((reinterpret_cast<uintptr_t>(d_ws) & 255) != 0 || *ws_bytes < need) return KVR_E_WORKSPACE;
    if (c.n_seqs == 0 || c.n_queries == 0) return KVR_OK;
    if (!d_q || !d_out || !c.d_cu_q || !c.d_cu_k) return KVR_E_NULL;
    if (c.n_keys > 0 && (!d_k || !d_k_rot || !d_v)) return KVR_E_NULL;
    p.q = rows(d_q, c.n_queries, q_token_stride, c.n_q_heads, q_head_stride, dtype);
    p.k = rows(d_k, c.n_keys, k_token_stride, c.n_kv_heads, k_head_stride, dtype);
    p.v = rows(d_v, c.n_keys, v_token_stride, c.n_kv_heads, v_head_stride, dtype);
    p.shared = rows(d_k_rot, c.n_keys, k_rot_stride, 1, 0, dtype);
    p.out = rows(d_out, c.n_queries, out_token_stride, c.n_q_heads, out_head_stride, dtype);
    const Rows *all[5] = {&p.q, &p.k, &p.v, &p.shared, &p.out};
    for (const Rows *r : all)
        if (!rows_aligned(*r)) return KVR_E_LAYOUT;
    for (int i = 1; i < 4; ++i)
        if (all[i]->token_stride > (1 << 24)) return KVR_E_LAYOUT;
    p.lse = d_lse;
    p.cu_q = c.d_cu_q;
    p.cu_k = c.d_cu_k;
    p.scale2 = scale_log2(scale);
    p.negate = scale < 0.0f;
    p.status = d_status;
    if (need) {
        const size_t cells = need / sizeof(float) / (size_t)(c.nope + 4);
        p.part_o = static_cast<float *>(d_ws);
        p.part_ml = reinterpret_cast<float4 *>(p.part_o + cells * (size_t)c.nope);
    }
    KVR_TRY(kvr::kv::launch_prompt(p, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

}  // extern "C"
