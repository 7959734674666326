// C ABI of the paged KV cache: validation on the host, frequencies of rotary
// positions, launches.
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "kvr.h"
#include "kvr_kv_host.h"

namespace {

using kvr::kv::Attention;
using kvr::kv::Cache;
using kvr::kv::Rotary;
using kvr::kv::Rows;

int check_cache(const kvr_kv_cache *c, Cache &out)
{
    if (!c) return KVR_E_NULL;
    if (c->format < KVR_KV_BF16 || c->format > KVR_KV_FP4) return KVR_E_LAYOUT;
    const bool quant = c->format == KVR_KV_FP8 || c->format == KVR_KV_FP4;
    if (!c->k_data || !c->v_data || (quant && (!c->k_scale || !c->v_scale))) return KVR_E_NULL;
    if (c->n_pages < 1 || c->n_pages > INT32_MAX || c->n_kv_heads < 1 || c->n_kv_heads > 1024)
        return KVR_E_SIZE;
    const int32_t ps = c->page_size;
    if (ps < 16 || ps > 32768 || (ps & (ps - 1)) != 0) return KVR_E_LAYOUT;
    const int32_t hd = c->head_dim;
    if (hd != 64 && hd != 96 && hd != 128 && hd != 192 && hd != 256) return KVR_E_LAYOUT;
    if (!aligned16(c->k_data) || !aligned16(c->v_data)) return KVR_E_LAYOUT;
    // strides of a single page or head do not matter
    const int64_t page = c->n_pages > 1 ? c->page_stride : 0;
    const int64_t head = c->n_kv_heads > 1 ? c->head_stride : 0;
    const int64_t spage = c->n_pages > 1 ? c->scale_page_stride : 0;
    const int64_t shead = c->n_kv_heads > 1 ? c->scale_head_stride : 0;
    const int64_t st[3] = {page, head, c->token_stride};
    for (int64_t s : st)
        if (s < 0 || s % 16 != 0) return KVR_E_LAYOUT;
    if (c->token_stride > (1 << 26)) return KVR_E_LAYOUT;
    if (quant && (spage < 0 || shead < 0 || c->scale_token_stride < 0 ||
                  c->scale_token_stride > (1 << 26)))
        return KVR_E_LAYOUT;
    out.k = static_cast<char *>(c->k_data);
    out.v = static_cast<char *>(c->v_data);
    out.ks = static_cast<uint8_t *>(c->k_scale);
    out.vs = static_cast<uint8_t *>(c->v_scale);
    out.page_stride = page;
    out.head_stride = head;
    out.token_stride = c->token_stride;
    out.spage_stride = spage;
    out.shead_stride = shead;
    out.stoken_stride = c->scale_token_stride;
    out.n_pages = c->n_pages;
    out.page_shift = __builtin_ctz((unsigned)ps);
    out.n_heads = c->n_kv_heads;
    out.dim = c->head_dim;
    out.format = c->format;
    return KVR_OK;
}

bool finite_from(double x, double low) { return std::isfinite(x) && x >= low; }

}  // namespace

extern "C" {

int kvr_rotary_table(const kvr_rope *rope, int32_t rot_dim, int64_t n_pos, float *d_table,
                     void *hip_stream)
{
    if (!rope || !d_table) return KVR_E_NULL;
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 2 * kvr::kv::kMaxFreq || n_pos < 0 ||
        n_pos > (int64_t(1) << 38) / rot_dim)
        return KVR_E_SIZE;
    if (rope->kind < KVR_ROPE_PLAIN || rope->kind > KVR_ROPE_INDEX) return KVR_E_METHOD;
    if (!std::isfinite(rope->theta) || !(rope->theta > 1.0)) return KVR_E_GRID;
    if (!std::isfinite(rope->magnitude) || !(rope->magnitude > 0.0)) return KVR_E_GRID;
    if (rope->kind != KVR_ROPE_PLAIN && !finite_from(rope->factor, 1.0)) return KVR_E_GRID;
    const bool blend = rope->kind == KVR_ROPE_TURNS || rope->kind == KVR_ROPE_INDEX;
    if (blend && (!std::isfinite(rope->low) || !std::isfinite(rope->high) || !(rope->low > 0.0) ||
                  !(rope->high > rope->low) || !std::isfinite(rope->trained_len) ||
                  !(rope->trained_len > 0.0)))
        return KVR_E_GRID;
    if (rope->kind == KVR_ROPE_BASE && rot_dim < 4) return KVR_E_SIZE;
    constexpr double kTwoPi = 6.283185307179586476925;
    double theta = rope->theta;
    if (rope->kind == KVR_ROPE_BASE)
        theta *= std::pow(rope->factor, (double)rot_dim / (rot_dim - 2));
    double a = 0.0, b = 1.0;
    if (rope->kind == KVR_ROPE_INDEX) {
        auto index = [&](double turns) {
            return rot_dim * std::log(rope->trained_len / (turns * kTwoPi)) /
                   (2.0 * std::log(theta));
        };
        a = std::fmin(std::fmax(std::floor(index(rope->high)), 0.0), rot_dim - 1.0);
        b = std::fmin(std::fmax(std::ceil(index(rope->low)), 0.0), rot_dim - 1.0);
        if (b <= a) b = a + 0.001;
    }
    kvr::kv::Freqs f{};
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double w = std::pow(theta, -2.0 * i / rot_dim);
        double keep = 1.0;   // share of the unchanged frequency
        if (rope->kind == KVR_ROPE_LINEAR) keep = 0.0;
        if (rope->kind == KVR_ROPE_TURNS)
            keep = (rope->trained_len * w / kTwoPi - rope->low) / (rope->high - rope->low);
        if (rope->kind == KVR_ROPE_INDEX) keep = 1.0 - (i - a) / (b - a);
        keep = std::fmin(std::fmax(keep, 0.0), 1.0);
        f.w[i] = keep >= 1.0 ? w : keep * w + (1.0 - keep) * (w / rope->factor);
    }
    if (n_pos == 0) return KVR_OK;
    KVR_TRY(kvr::kv::launch_rotary_table(f, rope->magnitude, rot_dim, n_pos, d_table,
                                         static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_rotary(const void *d_x, void *d_out, int32_t dtype, int64_t n_tokens, int32_t n_heads,
               int32_t head_dim, int64_t x_token_stride, int64_t x_head_stride,
               int64_t out_token_stride, int64_t out_head_stride, const int32_t *d_pos,
               const float *d_table, int64_t n_pos, int32_t rot_dim, int32_t flags,
               int32_t *d_status, void *hip_stream)
{
    if (n_tokens < 0 || n_heads < 1 || n_heads > 65536 || head_dim < 2 || head_dim > 4096 ||
        n_tokens > kMaxRows / n_heads)
        return KVR_E_SIZE;
    if (!dtype_ok(dtype)) return KVR_E_LAYOUT;
    Rotary r{};
    if (n_tokens == 0) return KVR_OK;
    if (!d_x || !d_out || !d_table) return KVR_E_NULL;
    int rc = check_rotary(d_pos, d_table, n_pos, rot_dim, head_dim, flags, r);
    if (rc != KVR_OK) return rc;
    const Rows x = rows(d_x, n_tokens, x_token_stride, n_heads, x_head_stride, dtype);
    const Rows out = rows(d_out, n_tokens, out_token_stride, n_heads, out_head_stride, dtype);
    if (x.token_stride < 0 || x.head_stride < 0 || out.token_stride < 0 || out.head_stride < 0)
        return KVR_E_LAYOUT;
    const uintptr_t odd = (uintptr_t)(dtype_bytes(dtype) - 1);
    if ((reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_out)) & odd)
        return KVR_E_LAYOUT;
    KVR_TRY(kvr::kv::launch_rotary(x, out, n_tokens, n_heads, head_dim, r, d_status,
                                   static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_cache_write(const kvr_kv_cache *cache, const void *d_k, const void *d_v, int32_t dtype,
                    int64_t n_tokens, int64_t k_token_stride, int64_t k_head_stride,
                    int64_t v_token_stride, int64_t v_head_stride, const int64_t *d_slots,
                    const int32_t *d_pos, const float *d_table, int64_t n_pos, int32_t rot_dim,
                    int32_t flags, int32_t *d_status, void *hip_stream)
{
    Cache c{};
    int rc = check_cache(cache, c);
    if (rc != KVR_OK) return rc;
    if (n_tokens < 0 || n_tokens > kMaxRows / c.n_heads) return KVR_E_SIZE;
    if (!dtype_ok(dtype)) return KVR_E_LAYOUT;
    if (n_tokens == 0) return KVR_OK;
    if (!d_k || !d_v || !d_slots) return KVR_E_NULL;
    Rotary r{};
    if (d_table) {
        rc = check_rotary(d_pos, d_table, n_pos, rot_dim, c.dim, flags, r);
        if (rc != KVR_OK) return rc;
    }
    const Rows k = rows(d_k, n_tokens, k_token_stride, c.n_heads, k_head_stride, dtype);
    const Rows v = rows(d_v, n_tokens, v_token_stride, c.n_heads, v_head_stride, dtype);
    if (!rows_aligned(k) || !rows_aligned(v)) return KVR_E_LAYOUT;
    KVR_TRY(kvr::kv::launch_cache_write(c, k, v, n_tokens, d_slots, r, d_status,
                                        static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_cache_read(const kvr_kv_cache *cache, const int64_t *d_slots, int64_t n_tokens, void *d_k,
                   void *d_v, int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                   int64_t v_token_stride, int64_t v_head_stride, int32_t *d_status,
                   void *hip_stream)
{
    Cache c{};
    const int rc = check_cache(cache, c);
    if (rc != KVR_OK) return rc;
    if (n_tokens < 0 || n_tokens > kMaxRows / c.n_heads) return KVR_E_SIZE;
    if (!dtype_ok(dtype)) return KVR_E_LAYOUT;
    if (n_tokens == 0) return KVR_OK;
    if (!d_k || !d_v || !d_slots) return KVR_E_NULL;
    const Rows k = rows(d_k, n_tokens, k_token_stride, c.n_heads, k_head_stride, dtype);
    const Rows v = rows(d_v, n_tokens, v_token_stride, c.n_heads, v_head_stride, dtype);
    if (!rows_aligned(k) || !rows_aligned(v)) return KVR_E_LAYOUT;
    KVR_TRY(kvr::kv::launch_cache_read(c, k, v, n_tokens, d_slots, d_status,
                                       static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_tree_attention(const kvr_kv_cache *cache, const kvr_sequences *seqs, const void *d_q,
                       int32_t dtype, int32_t n_q_heads, int64_t q_token_stride,
                       int64_t q_head_stride, const uint64_t *d_tree_mask, int32_t mask_words,
                       float scale, void *d_out, int64_t out_token_stride, int64_t out_head_stride,
                       float *d_lse, int32_t *d_status, void *d_ws, size_t *ws_bytes,
                       void *hip_stream)
{
    Attention a{};
    const int rc = check_cache(cache, a.c);
    if (rc != KVR_OK) return rc;
    if (!seqs || !ws_bytes) return KVR_E_NULL;
    if (dtype != KVR_DT_BF16 && dtype != KVR_DT_FP16) return KVR_E_LAYOUT;
    if ((a.c.format == KVR_KV_BF16 && dtype != KVR_DT_BF16) ||
        (a.c.format == KVR_KV_FP16 && dtype != KVR_DT_FP16))
        return KVR_E_LAYOUT;
    if (n_q_heads < a.c.n_heads || n_q_heads % a.c.n_heads != 0) return KVR_E_SIZE;
    if (seqs->n_seqs < 0 || seqs->n_seqs > kvr::kv::kMaxSeqs || seqs->max_q < 1 ||
        seqs->max_kv < 1 || seqs->max_kv > (1 << 30) || seqs->n_queries < 0 ||
        seqs->n_queries > INT32_MAX || seqs->max_pages < 0 || seqs->pages_stride < 0 ||
        (int64_t)seqs->max_q * n_q_heads > (1 << 24))
        return KVR_E_SIZE;
    if (d_tree_mask && (mask_words < 1 || (int64_t)mask_words * 64 < seqs->max_q)) return KVR_E_SIZE;
    if (!std::isfinite(scale)) return KVR_E_GRID;
    a.group = n_q_heads / a.c.n_heads;
    a.q_heads = n_q_heads;
    a.n_seqs = seqs->n_seqs;
    a.max_q = seqs->max_q;
    a.max_kv = seqs->max_kv;
    a.n_queries = seqs->n_queries;
    a.max_pages = seqs->max_pages;
    const size_t need = kvr::kv::plan_attention(a);
    if (!d_ws) {
        *ws_bytes = need;
        return KVR_OK;
    }
    if ((reinterpret_cast<uintptr_t>(d_ws) & 255) != 0 || *ws_bytes < need) return KVR_E_WORKSPACE;
    if (seqs->n_seqs == 0 || seqs->n_queries == 0) return KVR_OK;
    if (!d_q || !d_out || !seqs->d_cu_q || !seqs->d_kv_len || !seqs->d_pages) return KVR_E_NULL;
    a.q = rows(d_q, a.n_queries, q_token_stride, n_q_heads, q_head_stride, dtype);
    a.out = rows(d_out, a.n_queries, out_token_stride, n_q_heads, out_head_stride, dtype);
    if (!rows_aligned(a.q) || !rows_aligned(a.out)) return KVR_E_LAYOUT;
    a.lse = d_lse;
    a.cu_q = seqs->d_cu_q;
    a.kv_len = seqs->d_kv_len;
    a.pages = seqs->d_pages;
    a.pages_stride = seqs->pages_stride;
    a.mask = d_tree_mask;
    a.words = mask_words;
    a.scale2 = (float)(std::fabs((double)scale) * 1.4426950408889634);
    if (a.scale2 == 0.0f) a.scale2 = FLT_MIN;   // keeps -infinity times it -infinity
    a.negate = scale < 0.0f;
    a.status = d_status;
    if (need) {
        const size_t cells = need / sizeof(float) / (size_t)(a.c.dim + 4);
        a.part_o = static_cast<float *>(d_ws);
        a.part_ml = reinterpret_cast<float4 *>(a.part_o + cells * (size_t)a.c.dim);
    }
    KVR_TRY(kvr::kv::launch_attention(a, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

}  // extern "C"
