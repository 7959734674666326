// C ABI of a cache's pages: validation on the host, workspaces, launches.
#include <algorithm>
#include <cstdint>

#include "kvr.h"
#include "kvr_kv_host.h"
#include "kvr_pages.h"

namespace {

using kvr::pages::Compact;
using kvr::pages::Copy;
using kvr::pages::Pool;
using kvr::pages::Resize;

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int check_pool(const kvr_page_pool *p, int32_t *status, Pool &out)
{
    if (!p) return KVR_E_NULL;
    if (p->n_pages < 1 || p->n_pages > (1 << 30) || p->n_seqs < 0 || p->n_seqs > 65536 ||
        p->max_pages < 0 || p->max_pages > (1 << 24) || p->pages_stride < 0)
        return KVR_E_SIZE;
    const int32_t ps = p->page_size;
    if (ps < 16 || ps > 32768 || (ps & (ps - 1)) != 0) return KVR_E_LAYOUT;
    if (p->n_seqs > 1 && p->pages_stride < p->max_pages) return KVR_E_LAYOUT;   // rows would share entries
    out.refs = p->d_refs;
    out.table = p->d_pages;
    out.len = p->d_kv_len;
    out.n_pages = p->n_pages;
    out.stride = p->pages_stride;
    out.width = p->max_pages;
    out.n_seqs = p->n_seqs;
    out.shift = __builtin_ctz((unsigned)ps);
    out.words = kvr::pages::chunk_words(p->n_pages);
    out.chunks = (int32_t)kvr::kv::cdiv(p->n_pages, 64 * (int64_t)out.words);
    out.status = status;
    return KVR_OK;
}
// Rows of no entries need no table.
bool complete(const Pool &p) { return p.refs && p.len && (p.table || p.width == 0); }

int check_workspace(void *d_ws, size_t *ws_bytes, size_t need)
{
    return (reinterpret_cast<uintptr_t>(d_ws) & 255) != 0 || *ws_bytes < need ? KVR_E_WORKSPACE : KVR_OK;
}

// The largest of 16, 4 and 1 that divides all of a tensor's addresses and sizes.
int32_t width_of(const kvr_page_buffer &b)
{
    const uint64_t all = reinterpret_cast<uintptr_t>(b.data) | (uint64_t)b.page_stride |
                         (uint64_t)(b.outer > 1 ? b.outer_stride : 0) |
                         (uint64_t)(b.inner > 1 ? b.inner_stride : 0) | (uint64_t)b.run_bytes;
    return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
}

// Runs that follow one another as one.
void merge(kvr_page_buffer &b)
{
    if (b.inner == 1 || b.inner_stride == b.run_bytes) {
        b.run_bytes *= b.inner;
        b.inner = 1;
        b.inner_stride = 0;
        if (b.outer > 1 && b.outer_stride == b.run_bytes) b.run_bytes *= b.outer, b.outer = 1;
    }
    if (b.inner > 1 && b.outer == 1) b.outer_stride = 0;
    if (b.inner == 1 && b.outer > 1) {   // one level
        b.inner = b.outer, b.inner_stride = b.outer_stride;
        b.outer = 1;
    }
    if (b.outer == 1) b.outer_stride = 0;
}

}  // namespace

extern "C" {

int kvr_pages_fork(const kvr_page_pool *pool, const int32_t *d_parent, int32_t *d_status,
                   void *hip_stream)
{
    Pool p{};
    const int rc = check_pool(pool, d_status, p);
    if (rc != KVR_OK) return rc;
    if (p.n_seqs == 0) return KVR_OK;
    if (!complete(p) || !d_parent) return KVR_E_NULL;
    KVR_TRY(kvr::pages::launch_fork(p, d_parent, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_pages_resize(const kvr_page_pool *pool, const int32_t *d_new_len, int32_t *d_copies,
                     int32_t *d_status, void *d_ws, size_t *ws_bytes, void *hip_stream)
{
    Resize r{};
    int rc = check_pool(pool, d_status, r.p);
    if (rc != KVR_OK) return rc;
    if (!ws_bytes) return KVR_E_NULL;
    const size_t free = (size_t)r.p.chunks * r.p.words * sizeof(uint64_t);
    const size_t count = round256((size_t)r.p.chunks * sizeof(int32_t));
    const size_t need = free + count + (size_t)r.p.n_seqs * sizeof(kvr::pages::Row);
    if (!d_ws) {
        *ws_bytes = need;
        return KVR_OK;
    }
    rc = check_workspace(d_ws, ws_bytes, need);
    if (rc != KVR_OK) return rc;
    if (r.p.n_seqs == 0) return KVR_OK;
    if (!complete(r.p) || !d_new_len || !d_copies) return KVR_E_NULL;
    r.new_len = d_new_len;
    r.copies = d_copies;
    char *ws = static_cast<char *>(d_ws);
    r.free = reinterpret_cast<uint64_t *>(ws);
    r.count = reinterpret_cast<int32_t *>(ws + free);
    r.rows = reinterpret_cast<kvr::pages::Row *>(ws + free + count);
    KVR_TRY(kvr::pages::launch_resize(r, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_pages_compact(const kvr_page_pool *pool, int32_t *d_moves, int64_t max_moves,
                      int32_t *d_used, int32_t *d_status, void *d_ws, size_t *ws_bytes,
                      void *hip_stream)
{
    Compact c{};
    int rc = check_pool(pool, d_status, c.p);
    if (rc != KVR_OK) return rc;
    if (!ws_bytes) return KVR_E_NULL;
    if (max_moves < 0 || max_moves > c.p.n_pages) return KVR_E_SIZE;
    const size_t free = (size_t)c.p.chunks * c.p.words * sizeof(uint64_t);
    const size_t count = round256((size_t)c.p.chunks * sizeof(int32_t));
    const size_t need = free + count + (size_t)c.p.n_pages * sizeof(int32_t);
    if (!d_ws) {
        *ws_bytes = need;
        return KVR_OK;
    }
    rc = check_workspace(d_ws, ws_bytes, need);
    if (rc != KVR_OK) return rc;
    if (!d_used || (max_moves > 0 && !d_moves) || !c.p.refs || (c.p.n_seqs > 0 && !complete(c.p)))
        return KVR_E_NULL;
    c.moves = d_moves;
    c.max_moves = max_moves;
    c.used = d_used;
    char *ws = static_cast<char *>(d_ws);
    c.free = reinterpret_cast<uint64_t *>(ws);
    c.count = reinterpret_cast<int32_t *>(ws + free);
    c.where = reinterpret_cast<int32_t *>(ws + free + count);
    KVR_TRY(kvr::pages::launch_compact(c, static_cast<hipStream_t>(hip_stream)));
    return KVR_OK;
}

int kvr_pages_copy(const kvr_page_buffer *buffers, int32_t n_buffers, int64_t n_pages,
                   const int32_t *d_pairs, int64_t n_pairs, int32_t *d_status, void *hip_stream)
{
    if (n_buffers < 0 || n_buffers > 65536 || n_pages < 1 || n_pages > INT32_MAX || n_pairs < 0 ||
        n_pairs > (1 << 30))
        return KVR_E_SIZE;
    if (n_buffers > 0 && !buffers) return KVR_E_NULL;
    for (int32_t i = 0; i < n_buffers; ++i) {
        const kvr_page_buffer &b = buffers[i];
        if (!b.data) return KVR_E_NULL;
        if (b.outer < 1 || b.inner < 1 || b.run_bytes < 1 ||
            b.run_bytes > (int64_t(1) << 40) / b.outer / b.inner)
            return KVR_E_SIZE;
        if (b.page_stride < 0 || b.outer_stride < 0 || b.inner_stride < 0) return KVR_E_LAYOUT;
    }
    if (n_pairs == 0 || n_buffers == 0) return KVR_OK;
    if (!d_pairs) return KVR_E_NULL;
    // Tensors whose pages are alike go together.
    for (int32_t i = 0; i < n_buffers;) {
        kvr_page_buffer b = buffers[i];
        const int32_t width = width_of(b);
        merge(b);
        Copy c{};
        c.page_stride = b.page_stride;
        c.outer = b.outer, c.outer_stride = b.outer_stride;
        c.inner = b.inner, c.inner_stride = b.inner_stride;
        c.run = b.run_bytes;
        c.width = width;
        c.n_pages = n_pages;
        c.pairs = d_pairs;
        c.n_pairs = n_pairs;
        c.status = d_status;
        while (i < n_buffers && c.n_buffers < kvr::pages::kBuffers) {
            kvr_page_buffer o = buffers[i];
            if (width_of(o) != width) break;
            merge(o);
            if (o.page_stride != c.page_stride || o.outer != c.outer || o.inner != c.inner ||
                o.outer_stride != c.outer_stride || o.inner_stride != c.inner_stride || o.run_bytes != c.run)
                break;
            c.data[c.n_buffers++] = static_cast<char *>(o.data);
            ++i;
        }
        // as many blocks a page as fill the GPU, with 4 KB or more each
        const int64_t bytes = c.run * c.outer * c.inner;
        c.split = (int32_t)std::max<int64_t>(
            1, std::min(2048 / (n_pairs * c.n_buffers), bytes / (256 * width)));
        KVR_TRY(kvr::pages::launch_copy(c, static_cast<hipStream_t>(hip_stream)));
    }
    return KVR_OK;
}

}  // extern "C"
