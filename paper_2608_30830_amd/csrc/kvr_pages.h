// Internal declarations of the pages of a cache: branches, lengths, compaction, copies.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvr.h"
#include "kvr_kv.h"

namespace kvr {
namespace pages {

// Free pages are the bits of words of 64.  A block counts `words` of them, a chunk: 8 to
// 65,536, so that the chunks are at most 2,048 (each block adds up all counts).
inline int chunk_words(int64_t n_pages)
{
    int words = 8;
    while (kv::cdiv(n_pages, 64 * (int64_t)words) > 2048) words *= 2;
    return words;
}
// Pools that one block goes through in one launch, for new lengths and for compaction.  (A call in a
// graph, one launch against two or three: new lengths of 32 rows in 1,024 pages 5.8 us against 6.8, of 64
// rows in 4,096 pages 8.0 against 7.3, of 16 in 16,384 15.1 against 8.6; compaction of 32 rows in 1,024 pages
// 5.3 against 8.4, of 64 in 4,096 7.1 against 8.6, of 160 9.3 against 8.8, of 64 in 16,384 12.9 against 8.9.)
constexpr int kSmallResize = 2048, kSmallSeqs = 1024, kSmallCompact = 4096, kFewSeqs = 64;
constexpr int kSmallEntries = 65536;   // of all rows of the table

struct Pool {
    int32_t *refs, *table, *len;
    int64_t n_pages, stride;
    int32_t width, n_seqs, shift;               // entries of a row; log2 of the page size
    int32_t words, chunks;                      // words of a chunk
    int *status;
};

// What a row of a resize call does.
struct Row {
    int64_t start;      // pages that the rows before it take
    int32_t take;       // pages that it takes
    int32_t first;      // entry of the first of them
    int32_t need;       // entries that it holds afterwards
    int32_t mode;
};

struct Resize {
    Pool p;
    const int32_t *new_len;
    int32_t *copies;
    uint64_t *free;     // [chunks * words] bits of the pages that are free
    int32_t *count;     // [chunks] of them
    Row *rows;          // [n_seqs]
};

struct Compact {
    Pool p;
    int32_t *moves, *used;
    int64_t max_moves;
    uint64_t *free;
    int32_t *count;
    int32_t *where;     // [n_pages] the move of a page beyond the used ones' number, or -1
};

constexpr int kBuffers = 64;   // of one launch
struct Copy {
    char *data[kBuffers];
    int64_t page_stride, outer_stride, inner_stride, run;   // bytes
    int32_t outer, inner, width;                            // width: bytes moved at a time
    int32_t n_buffers, split;                               // blocks of one page
    int64_t n_pages, n_pairs;
    const int32_t *pairs;
    int *status;
};

hipError_t launch_fork(const Pool &p, const int32_t *parent, hipStream_t stream);
hipError_t launch_resize(const Resize &r, hipStream_t stream);
hipError_t launch_compact(const Compact &c, hipStream_t stream);
hipError_t launch_copy(const Copy &c, hipStream_t stream);

}  // namespace pages
}  // namespace kvr
