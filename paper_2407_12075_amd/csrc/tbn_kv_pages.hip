// Pages of the key/value cache: bookkeeping (reserve, fork, release, compact) and data (copy, append, keep).
//
// Bookkeeping works on whole numbers, so its results depend on no order: allocation ranks the free pages by their
// numbers and the requests by (sequence, slot), counts that several sequences change are changed by atomic additions
// whose intermediate values nobody reads.  reserve and the listing half of compact need a count over all pages before
// they may write: one workgroup, 16384 pages per round of loads.
//
// Data calls are copies.  V is kept transposed (channel rows of `page` keys), so append turns its tile in LDS: rows of
// new values come in by 16 bytes per lane along the channels and leave by 16 bytes along the keys.
#include "tbn_kv.h"

namespace tbn {

namespace {

constexpr int kOne = 1024;               // threads of a one-workgroup kernel
constexpr int kOneWaves = kOne / kWave;
constexpr int kPer = 16;                 // pages per lane and round
constexpr int kRound = kOne * kPer;

// exclusive prefix of v over the workgroup's threads, and the total; `part` has kOneWaves words of LDS
__device__ __forceinline__ int64_t block_prefix(int64_t v, int64_t *part, int64_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    __syncthreads();   // part may still be read from the call before
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kOneWaves; ++w) {
        const int64_t p = part[w];
        before += w < wave ? p : 0;
        all += p;
    }
    total = all;
    return before + sum - v;
}

// Walks pages [begin, end) in rounds of kRound.  take(ref, page) says which pages count; the r-th of them (r from `rank`) goes to
// out(r, page).  Ends once `want` have been found.  Returns the number found.
template <typename Take, typename Out>
__device__ int rank_pages(const int32_t *refs, int begin, int end, int want, int64_t *part, Take take, Out out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0;
    for (int64_t at = begin; at < end && found < want; at += kRound) {
        const int64_t mine = at + wave * (kWave * kPer);
        int r[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int64_t i = mine + j * kWave + lane;
            r[j] = i < end ? refs[i] : -1;
        }
        uint64_t hit[kPer];
        int n = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int64_t i = mine + j * kWave + lane;
            hit[j] = __ballot(i < end && take(r[j]));
            n += __popcll(hit[j]);
        }
        __syncthreads();
        if (lane == 0) part[wave] = n;
        __syncthreads();
        int before = found, all = 0;
#pragma unroll
        for (int w = 0; w < kOneWaves; ++w) {
            const int p = static_cast<int>(part[w]);
            before += w < wave ? p : 0;
            all += p;
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if ((hit[j] >> lane) & 1) {
                const int rank = before + __popcll(hit[j] & ((uint64_t(1) << lane) - 1));
                if (rank < want) out(rank, static_cast<int>(mine + j * kWave + lane));
            }
            before += __popcll(hit[j]);
        }
        found += all;
    }
    return min(found, want);
}

// Three words of LDS per sequence: the last page it would write to (-1: none that is shared), its first fresh slot, the rank of its
// first fresh page.
__global__ __launch_bounds__(kOne) void kv_reserve_kernel(tbn_kv_index ix, const int32_t *__restrict__ n_new, int32_t *__restrict__ copy_src,
                                                          int32_t *__restrict__ copy_dst, int32_t *__restrict__ fresh) {
    extern __shared__ int lds[];
    __shared__ int64_t part[kOneWaves];
    __shared__ int bad;
    const int n = ix.n_seqs, tid = threadIdx.x, shift = __ffs(ix.page) - 1, n_pages = static_cast<int>(ix.n_pages);
    const int64_t most = int64_t(ix.max_pages) << shift;
    int *tail = lds, *first = lds + n, *rank = lds + 2 * n;
    if (tid == 0) bad = *ix.status;
    __syncthreads();
    int invalid = 0;
    for (int s = tid; s < n; s += kOne) {
        const int len = ix.lens[s], add = n_new[s];
        const bool ok = len >= 0 && add >= 0 && int64_t(len) + add <= most;
        invalid |= !ok;
        int t = -1;
        if (ok && add > 0 && (len & (ix.page - 1))) {
            t = page_in(ix.table[int64_t(s) * ix.max_pages + (len >> shift)], n_pages);
            if (ix.refs[t] <= 1) t = -1;
        }
        tail[s] = t;
        copy_src[s] = -1;
        copy_dst[s] = -1;
    }
    if (invalid) atomicCAS(&bad, 0, TBN_KV_INVALID);
    __syncthreads();
    if (bad) {
        if (tid == 0) *ix.status = bad;
        return;
    }
    int64_t total = 0;
    for (int s0 = 0; s0 < n; s0 += kOne) {
        const int s = s0 + tid;
        int64_t need = 0;
        if (s < n) {
            const int len = ix.lens[s], add = n_new[s], t = tail[s];
            int have = (len + ix.page - 1) >> shift;
            if (t >= 0) {   // shared: replaced while more than one owner is left
                int earlier = 0;
                for (int e = 0; e < s; ++e) earlier += tail[e] == t;
                if (ix.refs[t] - earlier > 1) --have;
            }
            first[s] = have;
            need = add > 0 ? ((int64_t(len) + add + ix.page - 1) >> shift) - have : 0;
        }
        int64_t all;
        const int64_t before = block_prefix(need, part, all);
        if (s < n) rank[s] = static_cast<int>(total + before);   // within the pool, or the call fails
        total += all;
        if (total > n_pages) break;
    }
    const int want = static_cast<int>(min(total, int64_t(n_pages)));
    const int found = total > n_pages ? 0 : rank_pages(ix.refs, 0, n_pages, want, part, [](int r) { return r == 0; },
                                                       [&](int r, int page) { fresh[r] = page; });
    if (found < total) {
        if (tid == 0) *ix.status = TBN_KV_FULL;
        return;
    }
    __syncthreads();
    for (int i = tid; i < total; i += kOne) {
        int lo = 0, hi = n - 1;   // the last sequence whose rank is at most i and that needs a page
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (rank[mid] <= i) lo = mid; else hi = mid - 1;
        }
        const int page = fresh[i];
        ix.table[int64_t(lo) * ix.max_pages + first[lo] + (i - rank[lo])] = page;
        ix.refs[page] = 1;
    }
    for (int s = tid; s < n; s += kOne) {
        const int len = ix.lens[s], add = n_new[s], t = tail[s];
        if (t >= 0 && first[s] < (len + ix.page - 1) >> shift) {
            copy_src[s] = t;
            copy_dst[s] = fresh[rank[s]];
            atomicSub(&ix.refs[t], 1);
        }
        if (add > 0) ix.lens[s] = len + add;
    }
}

__global__ __launch_bounds__(256) void kv_fork_kernel(tbn_kv_index ix, const int32_t *__restrict__ parents, const int32_t *__restrict__ children, int n) {
    const int i = blockIdx.x, tid = threadIdx.x, shift = __ffs(ix.page) - 1;
    const int from = parents[i], to = children[i];
    // pairs are judged one by one, by what no other pair of the call changes: nobody reads the row of a child that is let in
    int clash = 0;
    for (int j = tid; j < n; j += 256) clash |= (children[j] == to && j < i) || parents[j] == to;
    clash = __syncthreads_or(clash);
    const bool in = from >= 0 && from < ix.n_seqs && to >= 0 && to < ix.n_seqs;
    const int empty = in && !clash ? ix.lens[to] : -1;
    __syncthreads();   // every thread has read the child's length before it is written
    if (!in || clash || empty != 0) {
        if (tid == 0) atomicCAS(ix.status, 0, TBN_KV_INVALID);
        return;
    }
    const int len = len_in(ix.lens[from], int64_t(ix.max_pages) << shift), pages = (len + ix.page - 1) >> shift;
    const int32_t *src = ix.table + int64_t(from) * ix.max_pages;
    int32_t *dst = ix.table + int64_t(to) * ix.max_pages;
    for (int p = tid; p < pages; p += 256) {
        const int page = page_in(src[p], static_cast<int>(ix.n_pages));
        dst[p] = page;
        atomicAdd(&ix.refs[page], 1);
    }
    if (tid == 0) ix.lens[to] = len;
}

__global__ __launch_bounds__(256) void kv_release_kernel(tbn_kv_index ix, const int32_t *__restrict__ keep) {
    const int s = blockIdx.x, tid = threadIdx.x, shift = __ffs(ix.page) - 1;
    const int len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift);
    const int left = min(len, max(keep[s], 0));
    __syncthreads();   // every thread has read the length before it is written
    int32_t *row = ix.table + int64_t(s) * ix.max_pages;
    for (int p = ((left + ix.page - 1) >> shift) + tid; p < (len + ix.page - 1) >> shift; p += 256) {
        atomicSub(&ix.refs[page_in(row[p], static_cast<int>(ix.n_pages))], 1);
        row[p] = -1;
    }
    if (tid == 0) ix.lens[s] = left;
}

// ws: [0] pages in use, [1 + page] where a page goes
__global__ __launch_bounds__(kOne) void kv_compact_kernel(tbn_kv_index ix, int32_t *__restrict__ src, int32_t *__restrict__ dst, int32_t *__restrict__ count,
                                                          int32_t *__restrict__ ws) {
    __shared__ int64_t part[kOneWaves];
    const int tid = threadIdx.x, n_pages = static_cast<int>(ix.n_pages);
    int mine = 0;
    for (int64_t at = tid; at < n_pages; at += kRound) {
        int r[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) r[j] = at + j * kOne < n_pages ? ix.refs[at + j * kOne] : 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) mine += r[j] > 0;
    }
    int64_t in_use;
    (void)block_prefix(mine, part, in_use);
    const int used = static_cast<int>(in_use);
    const int most = static_cast<int>(n_pages / 2);
    const int n = rank_pages(ix.refs, used, n_pages, most, part, [](int r) { return r > 0; }, [&](int i, int page) { src[i] = page; });
    rank_pages(ix.refs, 0, used, n, part, [](int r) { return r <= 0; }, [&](int i, int page) { dst[i] = page; });
    __syncthreads();
    for (int i = tid; i < n; i += kOne) {
        const int a = src[i], b = dst[i];
        ws[1 + a] = b;
        ix.refs[b] = ix.refs[a];
        ix.refs[a] = 0;
    }
    if (tid == 0) {
        *count = n;
        ws[0] = used;
    }
}

__global__ __launch_bounds__(256) void kv_compact_table_kernel(tbn_kv_index ix, const int32_t *__restrict__ ws) {
    const int s = blockIdx.x, shift = __ffs(ix.page) - 1;
    const int used = ws[0], pages = (len_in(ix.lens[s], int64_t(ix.max_pages) << shift) + ix.page - 1) >> shift;
    int32_t *row = ix.table + int64_t(s) * ix.max_pages;
    for (int p = threadIdx.x; p < pages; p += 256) {
        const int page = row[p];
        if (page >= used && page < ix.n_pages) row[p] = ws[1 + page];
    }
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kPiece = 16384;   // bytes of a page's keys or values that a workgroup copies at a time

__global__ __launch_bounds__(256) void kv_copy_kernel(tbn_kv_pool p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int64_t n,
                                                      const int32_t *__restrict__ count, int page_bytes, int pieces) {
    if (count) n = min(n, static_cast<int64_t>(max(*count, 0)));
    const int per = 2 * pieces + (p.summary ? 1 : 0);
    for (int64_t item = blockIdx.x; item < n * per; item += gridDim.x) {
        const int64_t pair = item / per;
        const int what = static_cast<int>(item - pair * per), a = src[pair], b = dst[pair];
        if (a < 0 || b < 0 || a >= p.n_pages || b >= p.n_pages) continue;
        if (what < 2 * pieces) {
            char *base = static_cast<char *>(what < pieces ? p.k : p.v);
            const int at = (what < pieces ? what : what - pieces) * kPiece;
            const char *from = base + int64_t(a) * page_bytes + at;
            char *to = base + int64_t(b) * page_bytes + at;
            const int end = min(kPiece, page_bytes - at);
            u32x4_t w[kPiece / 4096];
#pragma unroll
            for (int j = 0; j < kPiece / 4096; ++j) {
                const int o = j * 4096 + threadIdx.x * 16;
                if (o < end) w[j] = *reinterpret_cast<const u32x4_t *>(from + o);
            }
#pragma unroll
            for (int j = 0; j < kPiece / 4096; ++j) {
                const int o = j * 4096 + threadIdx.x * 16;
                if (o < end) *reinterpret_cast<u32x4_t *>(to + o) = w[j];
            }
        } else {
            const int bytes = p.kv_heads * 2 * p.dim;
            for (int o = threadIdx.x * 16; o < bytes; o += 4096)
                *reinterpret_cast<u32x4_t *>(p.summary + int64_t(b) * bytes + o) = *reinterpret_cast<const u32x4_t *>(p.summary + int64_t(a) * bytes + o);
            for (int h = threadIdx.x; h < p.kv_heads; h += 256) p.step[int64_t(b) * p.kv_heads + h] = p.step[int64_t(a) * p.kv_heads + h];
        }
    }
}

// ---- append and keep: a workgroup of 256 threads per sequence, kv head and (append) page ---------------------------------------

constexpr int kThreads = 256;

template <typename T> struct Pack;   // 16 bytes of elements
template <> struct Pack<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void unpack(const u32x4_t &w, float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
    }
};
template <> struct Pack<uint16_t> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void unpack(const u32x4_t &w, float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};

struct SummaryLds {
    float hi[kThreads][9], lo[kThreads][9];   // 9: lanes that read one column of eight fall on different banks
    float most[kThreads / kWave];
    int bad;
};

// Summary of one page and kv head over its first `rows` rows (>= 1).  Lanes own 16 bytes of channels and every
// (256 / groups)-th row; partial extremes meet in LDS.  Every thread of the workgroup calls it.
template <typename T>
__device__ void summarize(const tbn_kv_pool &p, int64_t page, int head, int rows, SummaryLds &l) {
    constexpr int V = Pack<T>::kVec;
    const int tid = threadIdx.x, groups = p.dim / V, lanes = kThreads / groups;
    const int g = tid % groups, r0 = tid / groups;
    const T *k = static_cast<const T *>(p.k) + (page * p.kv_heads + head) * (int64_t(p.page) * p.dim);
    float hi[V], lo[V];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; ++i) hi[i] = -INFINITY, lo[i] = INFINITY;
    if (r0 < lanes)
        for (int r = r0; r < rows; r += lanes) {
            float f[V];
            Pack<T>::unpack(*reinterpret_cast<const u32x4_t *>(k + int64_t(r) * p.dim + g * V), f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                hi[i] = fmaxf(hi[i], f[i]);
                lo[i] = fminf(lo[i], f[i]);
                bad |= !(fabsf(f[i]) < INFINITY);
            }
        }
    __syncthreads();   // the arrays may still be read from the call before
    if (tid == 0) l.bad = 0;
    __syncthreads();
    if (bad) l.bad = 1;
    if (r0 < lanes)
#pragma unroll
        for (int i = 0; i < V; ++i) l.hi[tid][i] = hi[i], l.lo[tid][i] = lo[i];
    __syncthreads();
    float h = -INFINITY, m = INFINITY, a = 0.f;
    if (tid < p.dim) {
        const int gg = tid / V, i = tid % V;
        for (int j = 0; j < min(lanes, rows); ++j) {
            h = fmaxf(h, l.hi[j * groups + gg][i]);
            m = fminf(m, l.lo[j * groups + gg][i]);
        }
        a = fmaxf(fabsf(h), fabsf(m));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) a = fmaxf(a, __shfl_xor(a, d));
    if ((tid & 63) == 0) l.most[tid >> 6] = a;
    __syncthreads();
    a = fmaxf(fmaxf(l.most[0], l.most[1]), fmaxf(l.most[2], l.most[3]));
    const bool all_finite = !l.bad;
    const int x = all_finite ? exponent_of(a) : 0;
    if (tid < p.dim) {
        int8_t *out = p.summary + (page * p.kv_heads + head) * (2 * p.dim) + tid;
        const float up = pow2_of(6 - x);   // exact, and so are the products
        out[0] = all_finite ? static_cast<int8_t>(ceilf(h * up)) : 0;
        out[p.dim] = all_finite ? static_cast<int8_t>(floorf(m * up)) : 0;
    }
    if (tid == 0) p.step[page * p.kv_heads + head] = all_finite ? pow2_of(x - 6) : INFINITY;
}

constexpr int kCols = 64;   // channels of V that a workgroup turns at a time

template <typename T>
struct AppendLds {
    T tile[kCols][128 + 16 / sizeof(T)];   // + 16 bytes: rows stay aligned for 16-byte reads and start on different banks
};

// Rows [r0, r1) of a page come from tokens tok .. of the call.  ALIGNED: 16-byte loads from k_new and v_new.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(tbn_kv_pool p, tbn_kv_index ix, const T *__restrict__ k_new, int64_t k_stride,
                                                             const T *__restrict__ v_new, int64_t v_stride, const int32_t *__restrict__ cu_new,
                                                             int total) {
    constexpr int V = Pack<T>::kVec;
    __shared__ union { AppendLds<T> v; SummaryLds s; } lds;
    const int tid = threadIdx.x, s = blockIdx.z, head = blockIdx.y, shift = __ffs(p.page) - 1;
    if (*ix.status != 0) return;
    const int t0 = max(cu_new[s], 0), n = min(cu_new[s + 1], total) - t0;
    const int len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift);
    if (n <= 0 || n > len) return;
    const int slot = ((len - n) >> shift) + blockIdx.x, base = slot << shift;
    if (base >= len) return;
    const int64_t page = page_in(ix.table[int64_t(s) * ix.max_pages + slot], static_cast<int>(p.n_pages));
    const int r0 = max(len - n - base, 0), r1 = min(len - base, p.page);
    const int tok = t0 + base + r0 - (len - n);   // of row r0
    const int64_t at = (page * p.kv_heads + head) * (int64_t(p.page) * p.dim);
    T *kp = static_cast<T *>(p.k) + at, *vp = static_cast<T *>(p.v) + at;
    const T *ks = k_new + tok * k_stride + head * p.dim, *vs = v_new + tok * v_stride + head * p.dim;
    const int rows = r1 - r0;
    if constexpr (ALIGNED) {
        const int groups = p.dim / V;
        for (int i = tid; i < rows * groups; i += kThreads) {
            const int r = i / groups, c = (i - r * groups) * V;
            *reinterpret_cast<u32x4_t *>(kp + (r0 + r) * p.dim + c) = *reinterpret_cast<const u32x4_t *>(ks + r * k_stride + c);
        }
    } else {
        for (int i = tid; i < rows * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim;
            kp[(r0 + r) * p.dim + c] = ks[r * k_stride + c];
        }
    }
    // few rows: element by element, no turn
    if (rows < V) {
        for (int i = tid; i < rows * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim;
            vp[c * p.page + r0 + r] = vs[r * v_stride + c];
        }
    } else {
        const int a0 = (r0 + V - 1) / V * V, a1 = r1 / V * V;   // rows that go out by 16 bytes
        for (int c0 = 0; c0 < p.dim; c0 += kCols) {
            const int cols = min(kCols, p.dim - c0);
            __syncthreads();
            if constexpr (ALIGNED) {
                const int groups = cols / V;
                for (int i = tid; i < rows * groups; i += kThreads) {
                    const int r = i / groups, c = (i - r * groups) * V;
                    union { u32x4_t w; T e[V]; } u;
                    u.w = *reinterpret_cast<const u32x4_t *>(vs + r * v_stride + c0 + c);
#pragma unroll
                    for (int e = 0; e < V; ++e) lds.v.tile[c + e][r0 + r] = u.e[e];
                }
            } else {
                for (int i = tid; i < rows * cols; i += kThreads) {
                    const int r = i / cols, c = i - r * cols;
                    lds.v.tile[c][r0 + r] = vs[r * v_stride + c0 + c];
                }
            }
            __syncthreads();
            const int groups = max(a1 - a0, 0) / V;
            for (int i = tid; i < cols * groups; i += kThreads) {
                const int c = i / groups, r = a0 + (i - c * groups) * V;
                *reinterpret_cast<u32x4_t *>(vp + (c0 + c) * p.page + r) = *reinterpret_cast<const u32x4_t *>(&lds.v.tile[c][r]);
            }
            const int head_rows = min(a0, r1) - r0, odd = head_rows + max(r1 - max(a1, a0), 0);
            for (int i = tid; i < cols * odd; i += kThreads) {
                const int c = i / odd, j = i - c * odd, r = j < head_rows ? r0 + j : max(a1, a0) + j - head_rows;
                vp[(c0 + c) * p.page + r] = lds.v.tile[c][r];
            }
        }
    }
    if (p.summary) {
        __syncthreads();   // the keys written above are read again, the tile's LDS is used again
        summarize<T>(p, page, head, r1, lds.s);
    }
}

constexpr int kKeepRows = 32;   // rows in registers and LDS between their loads and their stores

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(tbn_kv_pool p, tbn_kv_index ix, const int32_t *__restrict__ base, const int32_t *__restrict__ picks,
                                                           int width, const int32_t *__restrict__ counts) {
    __shared__ T tile[kKeepRows][kMaxDim];
    __shared__ SummaryLds sum;
    __shared__ int32_t from[kKeepRows];
    const int tid = threadIdx.x, s = blockIdx.y, head = blockIdx.x, shift = __ffs(p.page) - 1, inside = p.page - 1;
    if (*ix.status != 0) return;
    const int len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift), b = base[s];
    const int n = b < 0 || b > len ? 0 : min(min(counts[s], width), len - b);
    if (n <= 0) return;
    const int32_t *row = ix.table + int64_t(s) * ix.max_pages;
    const int n_pages = static_cast<int>(p.n_pages);
    auto page_of = [&](int key) { return (int64_t(page_in(row[key >> shift], n_pages)) * p.kv_heads + head) * (int64_t(p.page) * p.dim); };
    T *k = static_cast<T *>(p.k), *v = static_cast<T *>(p.v);
    // Picks ascend and are at or above their places, so a chunk's sources lie behind every target of the chunks before it.
    for (int j0 = 0; j0 < n; j0 += kKeepRows) {
        const int m = min(kKeepRows, n - j0);
        __syncthreads();
        if (tid < m) {
            const int pick = picks[int64_t(s) * width + j0 + tid];
            from[tid] = pick > j0 + tid && pick < len - b ? b + pick : -1;   // -1: stays where it is, or is not there
        }
        __syncthreads();
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim, f = from[r];
            if (f >= 0) tile[r][c] = k[page_of(f) + (f & inside) * p.dim + c];
        }
        __syncthreads();
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim, t = b + j0 + r;
            if (from[r] >= 0) k[page_of(t) + (t & inside) * p.dim + c] = tile[r][c];
        }
        __syncthreads();
        for (int i = tid; i < m * p.dim; i += kThreads) {   // neighbouring lanes on neighbouring keys of a channel
            const int c = i / m, r = i - c * m, f = from[r];
            if (f >= 0) tile[r][c] = v[page_of(f) + c * p.page + (f & inside)];
        }
        __syncthreads();
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int c = i / m, r = i - c * m, t = b + j0 + r;
            if (from[r] >= 0) v[page_of(t) + c * p.page + (t & inside)] = tile[r][c];
        }
    }
    if (p.summary) {
        __syncthreads();
        for (int slot = b >> shift; (slot << shift) < b + n; ++slot)
            summarize<T>(p, page_in(row[slot], n_pages), head, min(b + n - (slot << shift), p.page), sum);
    }
}

}  // namespace

tbn_status launch_kv_reserve(const tbn_kv_index &ix, const int32_t *n_new, int32_t *copy_src, int32_t *copy_dst, int32_t *ws, hipStream_t stream) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_reserve_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 12 * kMaxSeqs);
    if (attr != hipSuccess) {
        set_error("tbn_kv_reserve: %s", hipGetErrorString(attr));
        return TBN_ERR_DEVICE;
    }
    hipLaunchKernelGGL(kv_reserve_kernel, dim3(1), dim3(kOne), 12u * ix.n_seqs, stream, ix, n_new, copy_src, copy_dst, ws);
    return check_launch("tbn_kv_reserve");
}

tbn_status launch_kv_fork(const tbn_kv_index &ix, const int32_t *parents, const int32_t *children, int32_t n, hipStream_t stream) {
    hipLaunchKernelGGL(kv_fork_kernel, dim3(n), dim3(256), 0, stream, ix, parents, children, n);
    return check_launch("tbn_kv_fork");
}

tbn_status launch_kv_release(const tbn_kv_index &ix, const int32_t *keep, hipStream_t stream) {
    hipLaunchKernelGGL(kv_release_kernel, dim3(ix.n_seqs), dim3(256), 0, stream, ix, keep);
    return check_launch("tbn_kv_release");
}

tbn_status launch_kv_compact(const tbn_kv_index &ix, int32_t *src, int32_t *dst, int32_t *count, int32_t *ws, hipStream_t stream) {
    hipLaunchKernelGGL(kv_compact_kernel, dim3(1), dim3(kOne), 0, stream, ix, src, dst, count, ws);
    hipLaunchKernelGGL(kv_compact_table_kernel, dim3(ix.n_seqs), dim3(256), 0, stream, ix, ws);
    return check_launch("tbn_kv_compact");
}

tbn_status launch_kv_copy_pages(const tbn_kv_pool &p, const int32_t *src, const int32_t *dst, int64_t n, const int32_t *count, hipStream_t stream) {
    const int64_t bytes = int64_t(p.kv_heads) * p.page * p.dim * (p.dt == TBN_F32 ? 4 : 2);   // at most 2^27
    const int64_t pieces = (bytes + kPiece - 1) / kPiece, items = n * (2 * pieces + 1);
    const unsigned grid = static_cast<unsigned>(items < 4096 ? items : 4096);
    hipLaunchKernelGGL(kv_copy_kernel, dim3(grid), dim3(256), 0, stream, p, src, dst, n, count, static_cast<int>(bytes), static_cast<int>(pieces));
    return check_launch("tbn_kv_copy_pages");
}

template <typename T>
static void launch_append_typed(const tbn_kv_pool &p, const tbn_kv_index &ix, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                                const int32_t *cu_new, int total, int32_t max_new, hipStream_t stream) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new) | k_stride * sizeof(T) | v_stride * sizeof(T)) & 15u) == 0;
    // pages that max_new keys can touch: one more than they fill
    const dim3 grid((max_new + p.page - 2) / p.page + 1, p.kv_heads, ix.n_seqs);
    const T *k = static_cast<const T *>(k_new), *v = static_cast<const T *>(v_new);
    if (aligned) hipLaunchKernelGGL((kv_append_kernel<T, true>), grid, dim3(kThreads), 0, stream, p, ix, k, k_stride, v, v_stride, cu_new, total);
    else hipLaunchKernelGGL((kv_append_kernel<T, false>), grid, dim3(kThreads), 0, stream, p, ix, k, k_stride, v, v_stride, cu_new, total);
}

tbn_status launch_kv_append(const tbn_kv_pool &p, const tbn_kv_index &ix, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                            const int32_t *cu_new, int64_t total, int32_t max_new, hipStream_t stream) {
    if (p.dt == TBN_F32) launch_append_typed<float>(p, ix, k_new, k_stride, v_new, v_stride, cu_new, static_cast<int>(total), max_new, stream);
    else launch_append_typed<uint16_t>(p, ix, k_new, k_stride, v_new, v_stride, cu_new, static_cast<int>(total), max_new, stream);
    return check_launch("tbn_kv_append");
}

tbn_status launch_kv_keep(const tbn_kv_pool &p, const tbn_kv_index &ix, const int32_t *base, const int32_t *picks, int32_t width, const int32_t *counts,
                          hipStream_t stream) {
    const dim3 grid(p.kv_heads, ix.n_seqs);
    if (p.dt == TBN_F32) hipLaunchKernelGGL((kv_keep_kernel<float>), grid, dim3(kThreads), 0, stream, p, ix, base, picks, width, counts);
    else hipLaunchKernelGGL((kv_keep_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, p, ix, base, picks, width, counts);
    return check_launch("tbn_kv_keep");
}

}  // namespace tbn
