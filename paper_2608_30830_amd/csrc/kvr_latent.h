// Internal declarations of the latent cache: one row a token for all heads, `rank`
// elements of latent and `rot` of a shared, rotated key.
#pragma once

#include "kvr_kv.h"

namespace kvr {
namespace kv {

// A latent cache as the kernels see it: byte strides, the page size as a shift.
struct Latents {
    char *rows;
    uint8_t *scale;
    int64_t page_stride, token_stride;      // bytes
    int64_t spage_stride, stoken_stride;    // bytes
    int64_t n_pages;
    int32_t page_shift, rank, rot, format;
};

struct LatentWrite {
    Latents c;
    Rows latent, key;       // [tokens][1][rank], [tokens][1][rot]
    const char *norm;       // [rank] in the type of the latents, or nullptr
    float eps;
    Rotary r;
    const int64_t *slots;
    uint32_t tokens;
    int *status;
};
hipError_t launch_latent_write(const LatentWrite &a, hipStream_t stream);

struct LatentRead {
    Latents c;
    Rows out;               // [tokens][1][rank + rot]
    const int64_t *slots;
    uint32_t tokens;
    int *status;
};
hipError_t launch_latent_read(const LatentRead &a, hipStream_t stream);

// Attention over the latents.  `a` describes it as attention with one KV head whose values
// have `rank` elements (kvr_kv.h); its cache has no pointers, only the pool and page sizes.
struct LatentAttention {
    Attention a;
    Latents c;
    int32_t span;   // row blocks of a part, about
};
// Fills the launch plan; returns the workspace bytes (0: no sequence is cut).
size_t plan_latent_attention(LatentAttention &l);
hipError_t launch_latent_attention(const LatentAttention &l, hipStream_t stream);
// The kernel by cache format.
hipError_t launch_latent_bf16(const LatentAttention &l, dim3 grid, hipStream_t stream);
hipError_t launch_latent_fp16(const LatentAttention &l, dim3 grid, hipStream_t stream);
hipError_t launch_latent_fp8(const LatentAttention &l, dim3 grid, hipStream_t stream);

// Prompts: keys and values of each head, and the rotated part that the heads share.
struct Prompt {
    Rows q, k, v, shared, out;   // shared: [keys][1][rot]
    float *lse;                  // [n_queries][q_heads] or nullptr
    const int32_t *cu_q, *cu_k;
    int64_t n_queries, n_keys;
    int32_t n_seqs, max_q, max_k, q_heads, kv_heads, group, nope, rot, causal;
    float scale2;                // |softmax scale| * log2(e)
    int32_t negate;              // the scale is negative: queries change sign
    // launch plan
    int32_t block_rows;          // queries of one block
    int32_t max_items;           // blocks of queries, of all sequences, at most
    int32_t parts;               // that each block's keys are cut into
    float *part_o;               // [parts][items][q_heads][block_rows][nope]
    float4 *part_ml;             // [parts][items][q_heads][block_rows]
    int *status;
};
// Fills the launch plan; returns the workspace bytes (0: nothing is cut).
size_t plan_prompt(Prompt &p);
hipError_t launch_prompt(const Prompt &p, hipStream_t stream);

}  // namespace kv
}  // namespace kvr
