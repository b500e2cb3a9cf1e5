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

// exclusive prefix of v (below 2^26) over the workgroup's threads, and the total; `part` has kOneWaves words of LDS
__device__ __forceinline__ int64_t block_prefix(uint32_t v, int64_t *part, int64_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t low = prefix_of_lanes(v & 0xffffu), high = prefix_of_lanes(v >> 16);
    const int64_t sum = int64_t(low) + (int64_t(high) << 16);
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

// A round's pages: lane l of wave w has page at + 1024 w + 64 j + l in r[j], -1 beyond `end`.
__device__ __forceinline__ void load_round(const int32_t *refs, int64_t at, int end, int (&r)[kPer]) {
    const int64_t mine = at + (threadIdx.x >> 6) * (kWave * kPer) + (threadIdx.x & 63);
#pragma unroll
    for (int j = 0; j < kPer; ++j) r[j] = mine + j * kWave < end ? refs[mine + j * kWave] : -1;
}

// Ranks the pages [begin, end) that take(ref) picks: the i-th of them goes to out(i, page), i < want; ends once they are found.  r holds
// the first round already.  Returns the number found, at most want.
template <typename Take, typename Out>
__device__ int rank_pages(const int32_t *refs, int begin, int end, int want, int64_t *part, int (&r)[kPer], Take take, Out out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0;
    for (int64_t at = begin; at < end && found < want; at += kRound) {
        const int64_t mine = at + wave * (kWave * kPer) + lane;
        if (at > begin) load_round(refs, at, end, r);
        uint64_t hit[kPer];
        int n = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            hit[j] = __ballot(mine + j * kWave < end && take(r[j]));
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
                if (rank < want) out(rank, static_cast<int>(mine + j * kWave));
            }
            before += __popcll(hit[j]);
        }
        found += all;
    }
    return min(found, want);
}

constexpr int kNear = 2048;   // of a list of pages, the part that stays in LDS

// Three words of LDS per sequence: the last page it would write to (-1: none that is shared), its first fresh slot, the rank of its
// first fresh page.  What nothing has to wait for (the first round of refs, status, the first 1024 sequences) is requested first.
__global__ __launch_bounds__(kOne) void kv_reserve_kernel(tbn_kv_index ix, const int32_t *__restrict__ n_new, int32_t *__restrict__ copy_src,
                                                          int32_t *__restrict__ copy_dst, int32_t *__restrict__ far) {
    extern __shared__ int lds[];
    __shared__ int64_t part[kOneWaves];
    __shared__ int near[kNear];
    const int n = ix.n_seqs, tid = threadIdx.x, shift = __ffs(ix.page) - 1, n_pages = static_cast<int>(ix.n_pages);
    const int64_t most = int64_t(ix.max_pages) << shift;
    int *tail = lds, *first = lds + n, *rank = lds + 2 * n;
    int r[kPer];
    load_round(ix.refs, 0, n_pages, r);
    const int before = *ix.status, len0 = tid < n ? ix.lens[tid] : 0, add0 = tid < n ? n_new[tid] : 0;
    bool invalid = false;
    for (int s = tid; s < n; s += kOne) {
        const int len = s == tid ? len0 : ix.lens[s], add = s == tid ? add0 : n_new[s];
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
    const bool any_invalid = __syncthreads_or(invalid);
    if (before || any_invalid) {
        if (tid == 0 && !before) *ix.status = TBN_KV_INVALID;
        return;
    }
    int64_t total = 0;
    for (int s0 = 0; s0 < n; s0 += kOne) {
        const int s = s0 + tid;
        uint32_t need = 0;   // at most max_pages, 2^25
        if (s < n) {
            const int len = s0 == 0 ? len0 : ix.lens[s], add = s0 == 0 ? add0 : n_new[s], t = tail[s];
            int have = (len + ix.page - 1) >> shift;
            if (t >= 0) {   // shared: replaced while more than one owner is left
                int earlier = 0;
#pragma unroll 8
                for (int e = 0; e < s; ++e) earlier += tail[e] == t;
                if (ix.refs[t] - earlier > 1) --have;
            }
            first[s] = have;
            need = add > 0 ? static_cast<uint32_t>(((int64_t(len) + add + ix.page - 1) >> shift) - have) : 0;
        }
        int64_t all;
        const int64_t mine = block_prefix(need, part, all);
        if (s < n) rank[s] = static_cast<int>(total + mine);   // within the pool, or the call fails
        total += all;
        if (total > n_pages) break;
    }
    const int want = static_cast<int>(min(total, int64_t(n_pages)));
    const int found = total > n_pages ? 0 : rank_pages(ix.refs, 0, n_pages, want, part, r, [](int x) { return x == 0; }, [&](int i, int page) {
        if (i < kNear) near[i] = page;
        else far[i] = page;
    });
    if (found < total) {
        if (tid == 0) *ix.status = TBN_KV_FULL;
        return;
    }
    __syncthreads();
    auto fresh = [&](int i) { return i < kNear ? near[i] : far[i]; };
    for (int i = tid; i < want; i += kOne) {
        int lo = 0, hi = n - 1;   // the last sequence whose rank is at most i and that needs a page
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (rank[mid] <= i) lo = mid; else hi = mid - 1;
        }
        const int page = fresh(i);
        ix.table[int64_t(lo) * ix.max_pages + first[lo] + (i - rank[lo])] = page;
        ix.refs[page] = 1;
    }
    for (int s = tid; s < n; s += kOne) {
        const int len = s == tid ? len0 : ix.lens[s], add = s == tid ? add0 : n_new[s], t = tail[s];
        if (t >= 0 && first[s] < (len + ix.page - 1) >> shift) {
            copy_src[s] = t;
            copy_dst[s] = fresh(rank[s]);
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
    __shared__ int near[2][kNear];   // the first sources and targets
    const int tid = threadIdx.x, n_pages = static_cast<int>(ix.n_pages);
    int r[kPer];
    uint32_t mine = 0;
    for (int64_t at = 0; at < n_pages; at += kRound) {
        load_round(ix.refs, at, n_pages, r);
#pragma unroll
        for (int j = 0; j < kPer; ++j) mine += r[j] > 0;
    }
    int64_t in_use;
    (void)block_prefix(mine, part, in_use);
    const int used = static_cast<int>(in_use), most = static_cast<int>(n_pages / 2);
    // a pool of one round is in r already: pages before `used` are left out by their numbers
    const bool one = n_pages <= kRound;
    int n;
    {
        const int begin = one ? 0 : used;
        const int64_t lane_at = (tid >> 6) * (kWave * kPer) + (tid & 63);
        int x[kPer];
        if (!one) load_round(ix.refs, begin, n_pages, x);
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = one ? (lane_at + j * kWave >= used ? r[j] : 0) : x[j];
        n = rank_pages(ix.refs, begin, n_pages, most, part, x, [](int v) { return v > 0; }, [&](int i, int page) {
            src[i] = page;
            if (i < kNear) near[0][i] = page;
        });
        if (!one) load_round(ix.refs, 0, used, r);
        rank_pages(ix.refs, 0, used, n, part, r, [](int v) { return v <= 0; }, [&](int i, int page) {
            dst[i] = page;
            if (i < kNear) near[1][i] = page;
        });
    }
    __syncthreads();
    for (int i = tid; i < n; i += kOne) {
        const int a = i < kNear ? near[0][i] : src[i], b = i < kNear ? near[1][i] : dst[i];
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
// row_at(r): where row r is.
template <typename T, typename Row>
__device__ void summarize(const tbn_kv_pool &p, int64_t page, int head, int rows, SummaryLds &l, Row row_at) {
    constexpr int V = Pack<T>::kVec;
    const int tid = threadIdx.x, groups = p.dim / V, lanes = kThreads / groups;
    const int g = tid % groups, r0 = tid / groups;
    float hi[V], lo[V];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; ++i) hi[i] = -INFINITY, lo[i] = INFINITY;
    if (r0 < lanes)
#pragma unroll 4
        for (int r = r0; r < rows; r += lanes) {
            float f[V];
            Pack<T>::unpack(*reinterpret_cast<const u32x4_t *>(row_at(r) + g * V), f);
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

// + 8 bytes: rows stay aligned for 8-byte reads, and lanes that write one channel of eight begin on different banks
template <typename T>
struct AppendLds {
    T tile[kCols][128 + 8 / sizeof(T)];
};

// Rows [r0, r1) of a page come from tokens tok .. of the call.  ALIGNED: 16-byte loads from k_new and v_new.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(tbn_kv_pool p, tbn_kv_index ix, const T *__restrict__ k_new, int64_t k_stride,
                                                             const T *__restrict__ v_new, int64_t v_stride, const int32_t *__restrict__ cu_new,
                                                             int total) {
    constexpr int V = Pack<T>::kVec;
    __shared__ union { AppendLds<T> v; SummaryLds s; } lds;
    const int tid = threadIdx.x, s = blockIdx.z, head = blockIdx.y, shift = __ffs(p.page) - 1;
    int t0;
    const int failed = *ix.status, n = tokens_in(cu_new, s, total, t0);
    const int len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift);
    if (failed || n <= 0 || n > len) return;
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
                // two rows at a time where elements are half a word: whole words go to LDS
                constexpr int kRows = 4 / sizeof(T);
                const int groups = cols / V, even = r0 & (kRows - 1), pairs = (rows + even + kRows - 1) / kRows;
                for (int i = tid; i < pairs * groups; i += kThreads) {
                    const int pr = i / groups, c = (i - pr * groups) * V, r = pr * kRows - even;   // from row r0 + r on
                    union Piece { u32x4_t w; T e[V]; } u[kRows];
#pragma unroll
                    for (int x = 0; x < kRows; ++x) u[x].w = *reinterpret_cast<const u32x4_t *>(vs + min(max(r + x, 0), rows - 1) * v_stride + c0 + c);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if constexpr (kRows == 2)   // rows before r0 and behind r1 get something that nobody reads
                            *reinterpret_cast<uint32_t *>(&lds.v.tile[c + e][r0 + r]) = u[0].e[e] | static_cast<uint32_t>(u[1].e[e]) << 16;
                        else
                            lds.v.tile[c + e][r0 + r] = u[0].e[e];
                    }
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
                union { u32x4_t w; uint2 h[2]; } u;
                u.h[0] = *reinterpret_cast<const uint2 *>(&lds.v.tile[c][r]);
                u.h[1] = *reinterpret_cast<const uint2 *>(&lds.v.tile[c][r + V / 2]);
                *reinterpret_cast<u32x4_t *>(vp + (c0 + c) * p.page + r) = u.w;
            }
            const int head_rows = min(a0, r1) - r0, odd = head_rows + max(r1 - max(a1, a0), 0);
            for (int i = tid; i < cols * odd; i += kThreads) {
                const int c = i / odd, j = i - c * odd, r = j < head_rows ? r0 + j : max(a1, a0) + j - head_rows;
                vp[(c0 + c) * p.page + r] = lds.v.tile[c][r];
            }
        }
    }
    if (p.summary) {
        __syncthreads();   // the tile's LDS is used again, and (not ALIGNED) the keys written above are read again
        summarize<T>(p, page, head, r1, lds.s, [&](int r) { return ALIGNED && r >= r0 ? ks + (r - r0) * k_stride : kp + r * p.dim; });
    }
}

constexpr int kKeepRows = 32;    // rows of keys and of values between their loads and their stores
constexpr int kKeepPages = 64;   // pages from the base's on whose numbers are at hand

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(tbn_kv_pool p, tbn_kv_index ix, const int32_t *__restrict__ base, const int32_t *__restrict__ picks,
                                                           int width, const int32_t *__restrict__ counts) {
    __shared__ union { T tile[2][kKeepRows][kMaxDim]; SummaryLds sum; } lds;
    __shared__ int32_t from[kKeepRows], pages[kKeepPages];
    const int tid = threadIdx.x, s = blockIdx.y, head = blockIdx.x, shift = __ffs(p.page) - 1, inside = p.page - 1;
    const int failed = *ix.status, len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift), b = base[s];
    const int n = b < 0 || b > len ? 0 : min(min(counts[s], width), len - b);
    if (failed || n <= 0) return;
    const int32_t *row = ix.table + int64_t(s) * ix.max_pages;
    const int n_pages = static_cast<int>(p.n_pages), slot0 = b >> shift, slots = ((len + inside) >> shift) - slot0;
    for (int i = tid; i < min(slots, kKeepPages); i += kThreads) pages[i] = page_in(row[slot0 + i], n_pages);
    auto page_at = [&](int slot) { return slot - slot0 < kKeepPages ? pages[slot - slot0] : page_in(row[slot], n_pages); };
    auto page_of = [&](int key) { return (int64_t(page_at(key >> shift)) * p.kv_heads + head) * (int64_t(p.page) * p.dim); };
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
#pragma unroll 4
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim, f = from[r];
            if (f >= 0) lds.tile[0][r][c] = k[page_of(f) + (f & inside) * p.dim + c];
        }
#pragma unroll 4
        for (int i = tid; i < m * p.dim; i += kThreads) {   // neighbouring lanes on neighbouring keys of a channel
            const int c = i / m, r = i - c * m, f = from[r];
            if (f >= 0) lds.tile[1][r][c] = v[page_of(f) + c * p.page + (f & inside)];
        }
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int r = i / p.dim, c = i - r * p.dim, t = b + j0 + r;
            if (from[r] >= 0) k[page_of(t) + (t & inside) * p.dim + c] = lds.tile[0][r][c];
        }
#pragma unroll 4
        for (int i = tid; i < m * p.dim; i += kThreads) {
            const int c = i / m, r = i - c * m, t = b + j0 + r;
            if (from[r] >= 0) v[page_of(t) + c * p.page + (t & inside)] = lds.tile[1][r][c];
        }
    }
    if (p.summary) {
        __syncthreads();
        for (int slot = b >> shift; (slot << shift) < b + n; ++slot) {
            const int64_t page = page_at(slot);
            const T *rows = k + (page * p.kv_heads + head) * (int64_t(p.page) * p.dim);
            summarize<T>(p, page, head, min(b + n - (slot << shift), p.page), lds.sum, [&](int r) { return rows + r * p.dim; });
        }
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
