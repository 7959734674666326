// Internal declarations of the paged KV cache's operators: rotary positions,
// quantised writes and reads, attention of drafted tokens over the cache.
// These sources are compiled with IEEE NaN handling: a cache holds whatever a
// model produced, and its unwritten rows hold whatever was in memory.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvr.h"

namespace kvr {
namespace kv {

constexpr int kBlock = 32;      // elements that share one scale byte
constexpr int kMinExp = -110;   // smallest block exponent: every value stays a normal number
constexpr int kBadScale = 255;  // scale byte of a block that held a NaN or an infinity

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Blocks in a row: a dimension of a launch holds at most 2^32 threads, so more blocks than
// these (of up to 256 threads) stand in the third dimension.
constexpr uint32_t kMaxGrid = 1u << 23;
inline dim3 grid_of(int64_t blocks, unsigned y = 1)
{
    return dim3((unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid), y, (unsigned)cdiv(blocks, kMaxGrid));
}

// Whether an output is written past the caches: more than the eight L2 of 4 MB hold, in
// rows of whole cache lines that one 16-byte store a lane fills.  Read of 131,072 tokens from
// 8 bits: 141 us against 159; of 32,749 from 4 bits: 27 against 30; rotary of 32,768 tokens,
// 32 heads of 128 in 16 bits: 101 against 104 (inputs in the cache: 89 against 105).  But
// 12.6 MB written and read again 21.7 against 19.6, rows of 192 bytes 31 against 29, and
// 32-bit outputs, two stores a lane, 102 against 60.
inline bool streams(int64_t elements, int dim, int32_t dtype)
{
    return dtype != KVR_DT_FP32 && dim % 64 == 0 && 2 * elements >= (32 << 20);
}

// A cache as the kernels see it: byte strides, the page size as a shift.
struct Cache {
    char *k, *v;
    uint8_t *ks, *vs;
    int64_t page_stride, head_stride, token_stride;      // bytes
    int64_t spage_stride, shead_stride, stoken_stride;   // bytes
    int64_t n_pages;
    int32_t page_shift, n_heads, dim, format;
};

// [tokens][heads][dim] activations: element strides, elements of a row adjacent.
struct Rows {
    char *p;
    int64_t token_stride, head_stride;
    int32_t dtype;
};

// cos and sin rows of the positions; t == nullptr: no rotation.
struct Rotary {
    const float *t;        // [n_pos][2][rot / 2]
    const int32_t *pos;    // [tokens]
    int64_t n_pos;
    int32_t rot;
    int32_t interleaved;
    float sign;            // of the sines: -1 for the adjoint
};

constexpr int kMaxFreq = 128;   // rot <= 256
struct Freqs {
    double w[kMaxFreq];
};

hipError_t launch_rotary_table(const Freqs &f, double magnitude, int rot, int64_t n_pos,
                               float *table, hipStream_t stream);
hipError_t launch_rotary(const Rows &x, const Rows &out, int64_t tokens, int heads, int dim,
                         const Rotary &r, int *status, hipStream_t stream);
hipError_t launch_cache_write(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                              const int64_t *slots, const Rotary &r, int *status,
                              hipStream_t stream);
hipError_t launch_cache_read(const Cache &c, const Rows &k, const Rows &v, int64_t tokens,
                             const int64_t *slots, int *status, hipStream_t stream);

constexpr int kStep = 32;        // cached tokens of one step of the attention loop
constexpr int kMaxSeqs = 4096;

struct Attention {
    Cache c;
    Rows q, out;                 // out.dtype == q.dtype
    float *lse;                  // [n_queries][q_heads] or nullptr
    const int32_t *cu_q, *kv_len, *pages;
    const uint64_t *mask;        // [n_queries][words] or nullptr (each token sees the ones before it)
    int64_t n_queries, pages_stride, max_pages;
    int32_t n_seqs, q_heads, group, max_q, max_kv, words;
    float scale2;                // |softmax scale| * log2(e)
    int32_t negate;              // the scale is negative: queries change sign
    // launch plan
    int32_t row_tiles;           // 16-row tiles of one wave
    int32_t shared;              // waves share cached tokens and divide rows (else the reverse)
    int32_t waves;               // of one block
    int32_t block_rows;          // rows of one block
    int32_t target;              // items (a part of a sequence x a block of rows) of one head, about
    int32_t max_items;           // bound on them
    int32_t min_steps;           // steps that a part has at least
    int32_t fit;                 // blocks that are resident at once, which the parts have to fit
                                 // (0: about `target` parts)
    int32_t direct;              // row blocks that each sequence has room for, where none is cut
                                 // and items are in order of sequences (0: items are searched)
    float *part_o;               // [items][heads][block_rows][dim]
    float4 *part_ml;             // [items][heads][block_rows]: maximum, sum of the weights, and
                                 // of the weights as rounded for the products
    int32_t *chosen;             // where the first block leaves the steps of a part for the joining
                                 // kernel (nullptr: that finds them itself)
    int *status;
};

// Fills the launch plan; returns the workspace bytes (0: no sequence is cut).
size_t plan_attention(Attention &a);
hipError_t launch_attention(const Attention &a, hipStream_t stream);
// Joins the parts that a call's workspace holds.
hipError_t launch_join(const Attention &a, hipStream_t stream);
// The attention kernel by cache format and query type.
hipError_t launch_attention_bf16(const Attention &a, dim3 grid, hipStream_t stream);
hipError_t launch_attention_fp16(const Attention &a, dim3 grid, hipStream_t stream);
hipError_t launch_attention_fp8(const Attention &a, dim3 grid, hipStream_t stream);    // bfloat16 q
hipError_t launch_attention_fp8h(const Attention &a, dim3 grid, hipStream_t stream);   // half q
hipError_t launch_attention_fp4(const Attention &a, dim3 grid, hipStream_t stream);
hipError_t launch_attention_fp4h(const Attention &a, dim3 grid, hipStream_t stream);

}  // namespace kv
}  // namespace kvr
