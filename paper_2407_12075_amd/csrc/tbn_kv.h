// Shared declarations of the paged key/value cache (tbn_kv_pages.hip, tbn_kv_attention.hip, tbn_kv_select.hip).
// Layout and meaning of the pool's and the index's arrays: include/tbn.h.
#pragma once
#include "tbn_common.h"

namespace tbn {

constexpr int kMaxSeqs = 8192;         // lists of tbn_kv_reserve in LDS
constexpr int kMaxDim = 256;
constexpr int kMaxSelect = 4096;
constexpr int64_t kMaxBlocks = int64_t(1) << 20;

struct KvQueries {     // the queries of an attention or selection call
    const void *q;
    int64_t q_stride;
    const int32_t *cu_q;
    int64_t total_q;
    int32_t max_q, heads;
    int64_t max_len;   // 1 .. max_pages * page
};

tbn_status launch_kv_reserve(const tbn_kv_index &ix, const int32_t *n_new, int32_t *copy_src, int32_t *copy_dst, int32_t *ws, hipStream_t stream);
tbn_status launch_kv_fork(const tbn_kv_index &ix, const int32_t *parents, const int32_t *children, int32_t n, hipStream_t stream);
tbn_status launch_kv_release(const tbn_kv_index &ix, const int32_t *keep, hipStream_t stream);
tbn_status launch_kv_compact(const tbn_kv_index &ix, int32_t *src, int32_t *dst, int32_t *count, int32_t *ws, hipStream_t stream);
tbn_status launch_kv_copy_pages(const tbn_kv_pool &p, const int32_t *src, const int32_t *dst, int64_t n, const int32_t *count, hipStream_t stream);
tbn_status launch_kv_append(const tbn_kv_pool &p, const tbn_kv_index &ix, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                            const int32_t *cu_new, int64_t total, int32_t max_new, hipStream_t stream);
tbn_status launch_kv_keep(const tbn_kv_pool &p, const tbn_kv_index &ix, const int32_t *base, const int32_t *picks, int32_t width,
                          const int32_t *counts, hipStream_t stream);

size_t tree_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q);
tbn_status launch_tree_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const uint32_t *mask,
                                 int32_t mask_words, float scale, float *ws, hipStream_t stream);
size_t block_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_select);
tbn_status launch_block_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const int32_t *picks,
                                  int32_t n_select, float scale, float *ws, hipStream_t stream);
size_t block_select_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q);
tbn_status launch_block_select(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t *picks, int32_t n_select, int32_t n_sink,
                               int32_t n_recent, uint32_t *ws, hipStream_t stream);

#if defined(__HIPCC__)

// what the GPU's data say is bounded before it becomes an address
__device__ __forceinline__ int32_t page_in(int32_t page, int32_t n_pages) { return min(max(page, 0), n_pages - 1); }
__device__ __forceinline__ int32_t len_in(int32_t len, int64_t most) { return min(max(len, 0), static_cast<int32_t>(most)); }

// exponent x with 2^(x-1) <= a < 2^x for finite a >= 0, at least -100; the power of two of a whole number -126 .. 127
__device__ __forceinline__ int exponent_of(float a) { return max(static_cast<int>(__float_as_uint(a) >> 23) - 126, -100); }
__device__ __forceinline__ float pow2_of(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }


// Sums over the lanes of a wave by data-parallel primitives: a step costs a few cycles, an exchange through LDS a hundred.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {   // 0 where no lane is read
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t prefix_of_lanes(uint32_t v) {   // inclusive
    v += from_lane<0x111, 0xf>(v);   // one, two, four, eight lanes up within rows of 16
    v += from_lane<0x112, 0xf>(v);
    v += from_lane<0x114, 0xf>(v);
    v += from_lane<0x118, 0xf>(v);
    v += from_lane<0x142, 0xa>(v);   // a row's last lane to the next row, the second row's to the upper half
    v += from_lane<0x143, 0xc>(v);
    return v;
}
#endif

}  // namespace tbn
