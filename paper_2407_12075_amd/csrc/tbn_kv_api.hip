// C ABI of the paged key/value cache and its attention: argument validation.  Contract of each entry point: include/tbn.h.
#include "tbn_kv.h"

using namespace tbn;

namespace {

// fn: NULL in the queries, which leave tbn_last_error alone
tbn_status fail(tbn_status st, const char *fn, const char *what) {
    if (fn) set_error("%s: %s", fn, what);
    return st;
}

bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool page_ok(int32_t page) { return page == 32 || page == 64 || page == 128; }

tbn_status check_index(const char *fn, const tbn_kv_index *ix) {
    if (!ix) return fail(TBN_ERR_NULL, fn, "index must not be NULL");
    if (!ix->table || !ix->lens || !ix->refs || !ix->status) return fail(TBN_ERR_NULL, fn, "table, lens, refs and status of the index must not be NULL");
    if (ix->n_seqs < 1 || ix->max_pages < 1 || ix->n_pages < 1 || ix->page < 1) return fail(TBN_ERR_SHAPE, fn, "sizes of the index must be positive");
    if (!page_ok(ix->page)) return fail(TBN_ERR_UNSUPPORTED, fn, "pages of 32, 64 or 128 keys");
    if (ix->n_seqs > kMaxSeqs || ix->n_pages > INT32_MAX || int64_t(ix->max_pages) * ix->page > (int64_t(1) << 30))
        return fail(TBN_ERR_UNSUPPORTED, fn, "at most 8192 sequences, 2^31 - 1 pages and 2^30 keys of a sequence");
    return TBN_OK;
}

tbn_status check_pool(const char *fn, const tbn_kv_pool *p) {
    if (!p) return fail(TBN_ERR_NULL, fn, "pool must not be NULL");
    if (!p->k || !p->v) return fail(TBN_ERR_NULL, fn, "k and v of the pool must not be NULL");
    if ((p->summary == nullptr) != (p->step == nullptr)) return fail(TBN_ERR_NULL, fn, "summary and step of the pool go together");
    if (p->dt != TBN_F32 && p->dt != TBN_BF16) return fail(TBN_ERR_UNSUPPORTED, fn, "unknown dtype");
    if (p->n_pages < 1 || p->kv_heads < 1 || p->dim < 1 || p->page < 1) return fail(TBN_ERR_SHAPE, fn, "sizes of the pool must be positive");
    if (!page_ok(p->page) || p->dim % 8 || p->dim > kMaxDim || p->kv_heads > 1024 || p->n_pages > INT32_MAX)
        return fail(TBN_ERR_UNSUPPORTED, fn, "pages of 32, 64 or 128 keys, dim a multiple of 8 up to 256, at most 1024 kv heads and 2^31 - 1 pages");
    if (!aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->summary, 16)) return fail(TBN_ERR_UNSUPPORTED, fn, "k, v and summary of the pool must be 16-byte aligned");
    return TBN_OK;
}

tbn_status check_workspace(const char *fn, size_t need, const void *ws, size_t bytes, unsigned to) {
    if (need && (!ws || bytes < need || !aligned(ws, to))) {
        set_error("%s: workspace of %zu bytes, %u-byte aligned, required (got %zu at %p)", fn, need, to, bytes, ws);
        return TBN_ERR_WORKSPACE;
    }
    return TBN_OK;
}

tbn_status check_pool(const char *fn, const tbn_kv4_pool *p) {
    if (!p) return fail(TBN_ERR_NULL, fn, "pool must not be NULL");
    if (!p->k || !p->v || !p->k_exp || !p->v_exp) return fail(TBN_ERR_NULL, fn, "k, v, k_exp and v_exp of the pool must not be NULL");
    if (p->n_pages < 1 || p->kv_heads < 1 || p->dim < 1 || p->page < 1) return fail(TBN_ERR_SHAPE, fn, "sizes of the pool must be positive");
    if (!page_ok(p->page) || p->dim % 32 || p->dim > kMaxDim || p->kv_heads > 1024 || p->n_pages > INT32_MAX)
        return fail(TBN_ERR_UNSUPPORTED, fn, "pages of 32, 64 or 128 keys, dim a multiple of 32 up to 256, at most 1024 kv heads and 2^31 - 1 pages");
    if (!aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->k_exp, 16) || !aligned(p->v_exp, 16))
        return fail(TBN_ERR_UNSUPPORTED, fn, "k, v, k_exp and v_exp of the pool must be 16-byte aligned");
    return TBN_OK;
}

template <typename Pool>
tbn_status check_both(const char *fn, const Pool *p, const tbn_kv_index *ix) {
    tbn_status st = check_pool(fn, p);
    if (st == TBN_OK) st = check_index(fn, ix);
    if (st == TBN_OK && (p->page != ix->page || p->n_pages != ix->n_pages)) st = fail(TBN_ERR_SHAPE, fn, "pool and index must agree on page and n_pages");
    return st;
}

tbn_status check_type(const char *fn, tbn_dtype dt) { return dt == TBN_F32 || dt == TBN_BF16 ? TBN_OK : fail(TBN_ERR_UNSUPPORTED, fn, "unknown dtype"); }

// pool, index, queries; max_len becomes 1 .. max_pages * page
template <typename Pool>
tbn_status check_queries(const char *fn, const Pool *p, const tbn_kv_index *ix, KvQueries &q) {
    const tbn_status st = check_both(fn, p, ix);
    if (st != TBN_OK) return st;
    const int64_t most = int64_t(ix->max_pages) * ix->page;
    if (q.total_q < 0 || q.max_q < 0 || q.heads < 1 || q.max_len < 0) return fail(TBN_ERR_SHAPE, fn, "total_q, max_q and max_len must be >= 0, heads positive");
    if (q.heads % p->kv_heads) return fail(TBN_ERR_SHAPE, fn, "heads must be a multiple of the pool's kv heads");
    if (q.heads > 65536 || q.total_q > (1 << 30)) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 65536 heads and 2^30 queries");
    if (q.max_len > most) return fail(TBN_ERR_SHAPE, fn, "max_len is beyond max_pages * page");
    if (q.max_len == 0) q.max_len = most;
    if (q.max_q > q.total_q) q.max_q = static_cast<int32_t>(q.total_q);
    return TBN_OK;
}

template <typename Pool>
tbn_status check_query_pointers(const char *fn, const Pool *p, const KvQueries &q, const void *out) {
    if (!q.q || !out || !q.cu_q) return fail(TBN_ERR_NULL, fn, "q, the output and cu_q must not be NULL");
    if (q.q_stride < int64_t(q.heads) * p->dim || q.q_stride > (int64_t(1) << 40)) return fail(TBN_ERR_SHAPE, fn, "q_stride must be at least heads * dim (and at most 2^40)");
    return TBN_OK;
}

// tokens of a call that appends to a pool or reads from it
tbn_status check_tokens(const char *fn, int64_t total, int32_t most) {
    if (total < 0 || most < 0) return fail(TBN_ERR_SHAPE, fn, "the number of tokens, all and of a sequence, must be >= 0");
    if (total > (1 << 30)) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 2^30 tokens");
    return TBN_OK;
}

template <typename Pool>
tbn_status check_strides(const char *fn, const Pool *pool, int64_t k_stride, int64_t v_stride) {
    const int64_t row = int64_t(pool->kv_heads) * pool->dim, lim = int64_t(1) << 40;
    if (k_stride < row || v_stride < row || k_stride > lim || v_stride > lim) return fail(TBN_ERR_SHAPE, fn, "k_stride and v_stride must be at least kv_heads * dim (and at most 2^40)");
    return TBN_OK;
}

int32_t least(int32_t a, int64_t b) { return a < b ? a : static_cast<int32_t>(b); }

}  // namespace

extern "C" {

size_t tbn_kv_workspace_bytes(int64_t n_pages, int32_t n_seqs) {
    if (n_pages < 1 || n_pages > INT32_MAX || n_seqs < 1 || n_seqs > kMaxSeqs) return 0;
    return 4 * (static_cast<size_t>(n_pages) + 1);
}

tbn_status tbn_kv_reserve(const tbn_kv_index *index, const int32_t *n_new, int32_t *copy_src, int32_t *copy_dst, void *workspace,
                          size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_kv_reserve";
    tbn_status st = check_index(fn, index);
    if (st != TBN_OK) return st;
    if (!n_new || !copy_src || !copy_dst) return fail(TBN_ERR_NULL, fn, "n_new, copy_src and copy_dst must not be NULL");
    st = check_workspace(fn, tbn_kv_workspace_bytes(index->n_pages, index->n_seqs), workspace, workspace_bytes, 4);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_kv_reserve(*index, n_new, copy_src, copy_dst, static_cast<int32_t *>(workspace), static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_fork(const tbn_kv_index *index, const int32_t *parents, const int32_t *children, int32_t n, void *stream) {
    const char *fn = "tbn_kv_fork";
    const tbn_status st = check_index(fn, index);
    if (st != TBN_OK) return st;
    if (n < 0 || n > index->n_seqs) return fail(TBN_ERR_SHAPE, fn, "n must be 0 .. n_seqs");
    if (n == 0) return TBN_OK;
    if (!parents || !children) return fail(TBN_ERR_NULL, fn, "parents and children must not be NULL");
    drop_stale_error();
    return launch_kv_fork(*index, parents, children, n, static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_release(const tbn_kv_index *index, const int32_t *keep, void *stream) {
    const char *fn = "tbn_kv_release";
    const tbn_status st = check_index(fn, index);
    if (st != TBN_OK) return st;
    if (!keep) return fail(TBN_ERR_NULL, fn, "keep must not be NULL");
    drop_stale_error();
    return launch_kv_release(*index, keep, static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_compact(const tbn_kv_index *index, int32_t *src, int32_t *dst, int32_t *count, void *workspace, size_t workspace_bytes,
                          void *stream) {
    const char *fn = "tbn_kv_compact";
    tbn_status st = check_index(fn, index);
    if (st != TBN_OK) return st;
    if (!count || (index->n_pages > 1 && (!src || !dst))) return fail(TBN_ERR_NULL, fn, "src, dst and count must not be NULL");
    st = check_workspace(fn, tbn_kv_workspace_bytes(index->n_pages, index->n_seqs), workspace, workspace_bytes, 4);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_kv_compact(*index, src, dst, count, static_cast<int32_t *>(workspace), static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_copy_pages(const tbn_kv_pool *pool, const int32_t *src, const int32_t *dst, int64_t n, const int32_t *count, void *stream) {
    const char *fn = "tbn_kv_copy_pages";
    const tbn_status st = check_pool(fn, pool);
    if (st != TBN_OK) return st;
    if (n < 0 || n > INT32_MAX) return fail(TBN_ERR_SHAPE, fn, "n must be 0 .. 2^31 - 1");
    if (n == 0) return TBN_OK;
    if (!src || !dst) return fail(TBN_ERR_NULL, fn, "src and dst must not be NULL");
    drop_stale_error();
    return launch_kv_copy_pages(*pool, src, dst, n, count, static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_append(const tbn_kv_pool *pool, const tbn_kv_index *index, const void *k_new, int64_t k_stride, const void *v_new,
                         int64_t v_stride, const int32_t *cu_new, int64_t total, int32_t max_new, void *stream) {
    const char *fn = "tbn_kv_append";
    tbn_status st = check_both(fn, pool, index);
    if (st != TBN_OK) return st;
    if ((st = check_tokens(fn, total, max_new)) != TBN_OK) return st;
    if (total == 0 || max_new == 0) return TBN_OK;
    if (!k_new || !v_new || !cu_new) return fail(TBN_ERR_NULL, fn, "k_new, v_new and cu_new must not be NULL");
    if ((st = check_strides(fn, pool, k_stride, v_stride)) != TBN_OK) return st;
    drop_stale_error();
    return launch_kv_append(*pool, *index, k_new, k_stride, v_new, v_stride, cu_new, total, least(max_new, total), static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv_keep(const tbn_kv_pool *pool, const tbn_kv_index *index, const int32_t *base, const int32_t *picks, int32_t width,
                       const int32_t *counts, void *stream) {
    const char *fn = "tbn_kv_keep";
    const tbn_status st = check_both(fn, pool, index);
    if (st != TBN_OK) return st;
    if (width < 0) return fail(TBN_ERR_SHAPE, fn, "width must be >= 0");
    if (width == 0) return TBN_OK;
    if (!base || !picks || !counts) return fail(TBN_ERR_NULL, fn, "base, picks and counts must not be NULL");
    drop_stale_error();
    return launch_kv_keep(*pool, *index, base, picks, width, counts, static_cast<hipStream_t>(stream));
}

size_t tbn_tree_attention_workspace_bytes(const tbn_kv_pool *pool, const tbn_kv_index *index, int64_t total_q, int32_t max_q, int32_t heads,
                                          int64_t max_len) {
    KvQueries q{nullptr, 0, nullptr, total_q, max_q, heads, max_len};
    if (check_queries(nullptr, pool, index, q) != TBN_OK || total_q == 0 || max_q == 0) return 0;
    return tree_attention_workspace(*pool, *index, q);
}

tbn_status tbn_tree_attention(const void *q, int64_t q_stride, void *out, float *lse, const tbn_kv_pool *pool, const tbn_kv_index *index,
                              const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t heads, const uint32_t *mask, int32_t mask_words,
                              int64_t max_len, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_tree_attention";
    KvQueries a{q, q_stride, cu_q, total_q, max_q, heads, max_len};
    tbn_status st = check_queries(fn, pool, index, a);
    if (st != TBN_OK) return st;
    if (mask && (mask_words < 0 || int64_t(mask_words) * 32 < max_q)) return fail(TBN_ERR_SHAPE, fn, "mask_words must hold max_q bits");
    if (total_q == 0 || max_q == 0) return TBN_OK;
    st = check_query_pointers(fn, pool, a, out);
    if (st == TBN_OK) st = check_workspace(fn, tree_attention_workspace(*pool, *index, a), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_tree_attention(*pool, *index, a, out, lse, mask, mask_words, scale, static_cast<float *>(workspace), static_cast<hipStream_t>(stream));
}

// n_sink and window of a call: nothing is beyond the longest sequence
static tbn_status check_window(const char *fn, const KvQueries &q, bool masked, int32_t &n_sink, int32_t &window) {
    if (n_sink < 0 || window < 1) return fail(TBN_ERR_SHAPE, fn, "n_sink must be >= 0, window positive");
    if (masked && q.max_q > window) return fail(TBN_ERR_SHAPE, fn, "with a mask the window must hold max_q tokens");
    constexpr int32_t kMost = 1 << 30;
    n_sink = n_sink < kMost ? n_sink : kMost;
    window = window < kMost ? window : kMost;
    return TBN_OK;
}

size_t tbn_window_attention_workspace_bytes(const tbn_kv_pool *pool, const tbn_kv_index *index, int64_t total_q, int32_t max_q, int32_t heads,
                                            int32_t n_sink, int32_t window, int32_t masked, int64_t max_len) {
    KvQueries q{nullptr, 0, nullptr, total_q, max_q, heads, max_len};
    if (check_queries(nullptr, pool, index, q) != TBN_OK || check_window(nullptr, q, masked != 0, n_sink, window) != TBN_OK || total_q == 0 || max_q == 0)
        return 0;
    return window_attention_workspace(*pool, *index, q, n_sink, window, masked != 0);
}

tbn_status tbn_window_attention(const void *q, int64_t q_stride, void *out, float *lse, const tbn_kv_pool *pool, const tbn_kv_index *index,
                                const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t heads, int32_t n_sink, int32_t window,
                                const uint32_t *mask, int32_t mask_words, int64_t max_len, float scale, void *workspace, size_t workspace_bytes,
                                void *stream) {
    const char *fn = "tbn_window_attention";
    KvQueries a{q, q_stride, cu_q, total_q, max_q, heads, max_len};
    tbn_status st = check_queries(fn, pool, index, a);
    if (st == TBN_OK) st = check_window(fn, a, mask != nullptr, n_sink, window);
    if (st != TBN_OK) return st;
    if (mask && (mask_words < 0 || int64_t(mask_words) * 32 < max_q)) return fail(TBN_ERR_SHAPE, fn, "mask_words must hold max_q bits");
    if (total_q == 0 || max_q == 0) return TBN_OK;
    st = check_query_pointers(fn, pool, a, out);
    if (st == TBN_OK) st = check_workspace(fn, window_attention_workspace(*pool, *index, a, n_sink, window, mask != nullptr), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_window_attention(*pool, *index, a, out, lse, n_sink, window, mask, mask_words, scale, static_cast<float *>(workspace),
                                   static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv4_append(const tbn_kv4_pool *pool, const tbn_kv_index *index, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                          tbn_dtype dt, const int32_t *cu_new, int64_t total, int32_t max_new, void *stream) {
    const char *fn = "tbn_kv4_append";
    tbn_status st = check_both(fn, pool, index);
    if (st == TBN_OK) st = check_type(fn, dt);
    if (st == TBN_OK) st = check_tokens(fn, total, max_new);
    if (st != TBN_OK || total == 0 || max_new == 0) return st;
    if (!k_new || !v_new || !cu_new) return fail(TBN_ERR_NULL, fn, "k_new, v_new and cu_new must not be NULL");
    if ((st = check_strides(fn, pool, k_stride, v_stride)) != TBN_OK) return st;
    drop_stale_error();
    return launch_kv4_append(*pool, *index, k_new, k_stride, v_new, v_stride, dt, cu_new, total, least(max_new, total), static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv4_read(const tbn_kv4_pool *pool, const tbn_kv_index *index, void *k_out, void *v_out, tbn_dtype dt, const int32_t *cu, int64_t total,
                        int32_t max_n, void *stream) {
    const char *fn = "tbn_kv4_read";
    tbn_status st = check_both(fn, pool, index);
    if (st == TBN_OK) st = check_type(fn, dt);
    if (st == TBN_OK) st = check_tokens(fn, total, max_n);
    if (st != TBN_OK || total == 0 || max_n == 0) return st;
    if (!k_out || !v_out || !cu) return fail(TBN_ERR_NULL, fn, "k_out, v_out and cu must not be NULL");
    drop_stale_error();
    return launch_kv4_read(*pool, *index, k_out, v_out, dt, cu, total, least(max_n, total), static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv4_copy_pages(const tbn_kv4_pool *pool, const int32_t *src, const int32_t *dst, int64_t n, const int32_t *count, void *stream) {
    const char *fn = "tbn_kv4_copy_pages";
    const tbn_status st = check_pool(fn, pool);
    if (st != TBN_OK) return st;
    if (n < 0 || n > INT32_MAX) return fail(TBN_ERR_SHAPE, fn, "n must be 0 .. 2^31 - 1");
    if (n == 0) return TBN_OK;
    if (!src || !dst) return fail(TBN_ERR_NULL, fn, "src and dst must not be NULL");
    drop_stale_error();
    return launch_kv4_copy_pages(*pool, src, dst, n, count, static_cast<hipStream_t>(stream));
}

tbn_status tbn_kv4_keep(const tbn_kv4_pool *pool, const tbn_kv_index *index, const int32_t *base, const int32_t *picks, int32_t width,
                        const int32_t *counts, void *stream) {
    const char *fn = "tbn_kv4_keep";
    const tbn_status st = check_both(fn, pool, index);
    if (st != TBN_OK) return st;
    if (width < 0) return fail(TBN_ERR_SHAPE, fn, "width must be >= 0");
    if (width == 0) return TBN_OK;
    if (!base || !picks || !counts) return fail(TBN_ERR_NULL, fn, "base, picks and counts must not be NULL");
    drop_stale_error();
    return launch_kv4_keep(*pool, *index, base, picks, width, counts, static_cast<hipStream_t>(stream));
}

// a call on the cache in 4 bits without a window passes with any n_sink
static tbn_status check_kv4(const char *fn, const tbn_kv4_pool *pool, const tbn_kv_index *index, tbn_dtype dt, KvQueries &q, bool masked, int32_t &n_sink,
                            int32_t &window) {
    tbn_status st = check_queries(fn, pool, index, q);
    if (st == TBN_OK) st = check_type(fn, dt);
    if (st == TBN_OK && window != 0) st = check_window(fn, q, masked, n_sink, window);
    return st;
}

size_t tbn_kv4_attention_workspace_bytes(const tbn_kv4_pool *pool, const tbn_kv_index *index, tbn_dtype dt, int64_t total_q, int32_t max_q, int32_t heads,
                                         int32_t n_sink, int32_t window, int32_t masked, int64_t max_len) {
    KvQueries q{nullptr, 0, nullptr, total_q, max_q, heads, max_len};
    if (check_kv4(nullptr, pool, index, dt, q, masked != 0, n_sink, window) != TBN_OK || total_q == 0 || max_q == 0) return 0;
    return kv4_attention_workspace(*pool, *index, q, dt, n_sink, window, masked != 0);
}

tbn_status tbn_kv4_attention(const void *q, int64_t q_stride, tbn_dtype dt, void *out, float *lse, const tbn_kv4_pool *pool, const tbn_kv_index *index,
                             const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t heads, int32_t n_sink, int32_t window, const uint32_t *mask,
                             int32_t mask_words, int64_t max_len, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_kv4_attention";
    KvQueries a{q, q_stride, cu_q, total_q, max_q, heads, max_len};
    tbn_status st = check_kv4(fn, pool, index, dt, a, mask != nullptr, n_sink, window);
    if (st != TBN_OK) return st;
    if (mask && (mask_words < 0 || int64_t(mask_words) * 32 < max_q)) return fail(TBN_ERR_SHAPE, fn, "mask_words must hold max_q bits");
    if (total_q == 0 || max_q == 0) return TBN_OK;
    st = check_query_pointers(fn, pool, a, out);
    if (st == TBN_OK) st = check_workspace(fn, kv4_attention_workspace(*pool, *index, a, dt, n_sink, window, mask != nullptr), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_kv4_attention(*pool, *index, a, dt, out, lse, n_sink, window, mask, mask_words, scale, static_cast<float *>(workspace),
                                static_cast<hipStream_t>(stream));
}

static tbn_status check_select(const char *fn, const tbn_kv_pool *pool, const tbn_kv_index *index, KvQueries &q) {
    const tbn_status st = check_queries(fn, pool, index, q);
    if (st != TBN_OK) return st;
    if (!pool->summary) return fail(TBN_ERR_NULL, fn, "the pool has no summary");
    if (q.heads / pool->kv_heads > 128) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 128 heads for a kv head");
    if (q.max_len > kMaxBlocks * pool->page) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 2^20 pages of a sequence");
    return TBN_OK;
}

size_t tbn_block_select_workspace_bytes(const tbn_kv_pool *pool, const tbn_kv_index *index, int64_t total_q, int32_t max_q, int32_t heads,
                                        int64_t max_len) {
    KvQueries q{nullptr, 0, nullptr, total_q, max_q, heads, max_len};
    if (check_select(nullptr, pool, index, q) != TBN_OK || total_q == 0 || max_q == 0) return 0;
    return block_select_workspace(*pool, *index, q);
}

tbn_status tbn_block_select(const void *q, int64_t q_stride, int32_t *picks, const tbn_kv_pool *pool, const tbn_kv_index *index,
                            const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t heads, int32_t n_select, int32_t n_sink,
                            int32_t n_recent, int64_t max_len, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_block_select";
    KvQueries a{q, q_stride, cu_q, total_q, max_q, heads, max_len};
    tbn_status st = check_select(fn, pool, index, a);
    if (st != TBN_OK) return st;
    if (n_select < 1 || n_sink < 0 || n_recent < 1 || int64_t(n_sink) + n_recent > n_select)
        return fail(TBN_ERR_SHAPE, fn, "n_sink >= 0, n_recent >= 1 and n_sink + n_recent <= n_select");
    if (n_select > kMaxSelect) return fail(TBN_ERR_UNSUPPORTED, fn, "n_select is at most 4096");
    if (total_q == 0 || max_q == 0) return TBN_OK;
    st = check_query_pointers(fn, pool, a, picks);
    if (st == TBN_OK) st = check_workspace(fn, block_select_workspace(*pool, *index, a), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_block_select(*pool, *index, a, picks, n_select, n_sink, n_recent, static_cast<uint32_t *>(workspace), static_cast<hipStream_t>(stream));
}

size_t tbn_block_attention_workspace_bytes(const tbn_kv_pool *pool, const tbn_kv_index *index, int64_t total_q, int32_t max_q, int32_t heads,
                                           int32_t n_select) {
    KvQueries q{nullptr, 0, nullptr, total_q, max_q, heads, 0};
    if (check_queries(nullptr, pool, index, q) != TBN_OK || total_q == 0 || max_q == 0 || n_select < 1 || n_select > kMaxSelect)
        return 0;
    return block_attention_workspace(*pool, *index, q, n_select);
}

tbn_status tbn_block_attention(const void *q, int64_t q_stride, void *out, float *lse, const tbn_kv_pool *pool, const tbn_kv_index *index,
                               const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t heads, const int32_t *picks, int32_t n_select,
                               float scale, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_block_attention";
    KvQueries a{q, q_stride, cu_q, total_q, max_q, heads, 0};
    tbn_status st = check_queries(fn, pool, index, a);
    if (st != TBN_OK) return st;
    if (n_select < 1) return fail(TBN_ERR_SHAPE, fn, "n_select must be positive");
    if (n_select > kMaxSelect) return fail(TBN_ERR_UNSUPPORTED, fn, "n_select is at most 4096");
    if (total_q == 0 || max_q == 0) return TBN_OK;
    if (!picks) return fail(TBN_ERR_NULL, fn, "picks must not be NULL");
    st = check_query_pointers(fn, pool, a, out);
    if (st == TBN_OK) st = check_workspace(fn, block_attention_workspace(*pool, *index, a, n_select), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_block_attention(*pool, *index, a, out, lse, picks, n_select, scale, static_cast<float *>(workspace), static_cast<hipStream_t>(stream));
}

static tbn_status check_verify(const char *fn, int64_t total, int32_t max_q, int32_t n_seqs, int64_t vocab) {
    if (total < 0 || max_q < 0 || n_seqs < 1 || vocab < 1) return fail(TBN_ERR_SHAPE, fn, "total_q and max_q must be >= 0, n_seqs and vocab positive");
    if (n_seqs > kMaxSeqs || total > (1 << 30) || vocab > (1 << 28)) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 8192 sequences, 2^30 tokens and a vocabulary of 2^28");
    return TBN_OK;
}

size_t tbn_verify_workspace_bytes(int64_t total_q, int32_t max_q, int32_t n_seqs, int64_t vocab) {
    if (check_verify(nullptr, total_q, max_q, n_seqs, vocab) != TBN_OK || max_q > verify_most_tokens()) return 0;
    return verify_workspace(total_q, max_q, n_seqs, vocab);
}

tbn_status tbn_verify(const float *target, int64_t target_stride, const float *draft, int64_t draft_stride, const int32_t *tokens, const int32_t *parents,
                      const float *u, const int32_t *cu_q, int64_t total_q, int32_t max_q, int32_t n_seqs, int64_t vocab, int32_t *picks, int32_t *counts,
                      int32_t *next, void *workspace, size_t workspace_bytes, void *stream) {
    const char *fn = "tbn_verify";
    tbn_status st = check_verify(fn, total_q, max_q, n_seqs, vocab);
    if (st != TBN_OK) return st;
    if (max_q > verify_most_tokens()) return fail(TBN_ERR_UNSUPPORTED, fn, "at most 2048 tokens of a sequence");
    if (!cu_q || !counts || !next || (max_q && !picks)) return fail(TBN_ERR_NULL, fn, "cu_q, picks, counts and next must not be NULL");
    if (total_q && max_q && (!target || !tokens || !u)) return fail(TBN_ERR_NULL, fn, "target, tokens and u must not be NULL");
    const int64_t lim = int64_t(1) << 40;
    if (target_stride < vocab || target_stride > lim || (draft && (draft_stride < vocab || draft_stride > lim)))
        return fail(TBN_ERR_SHAPE, fn, "target_stride and draft_stride must be at least vocab (and at most 2^40)");
    st = check_workspace(fn, verify_workspace(total_q, max_q, n_seqs, vocab), workspace, workspace_bytes, 16);
    if (st != TBN_OK) return st;
    drop_stale_error();
    return launch_verify(VerifyCall{target, draft, target_stride, draft_stride, tokens, parents, u, cu_q, total_q, max_q, n_seqs, vocab, picks, counts, next}, workspace,
                         static_cast<hipStream_t>(stream));
}

}  // extern "C"
