// Choice of cache pages for each query and kv head by the pages' summaries (definition: include/tbn.h).
//
//   score(b) = step_b * sum_d (pos_d max_b,d + neg_d min_b,d),  pos_d = sum_g max(c_gd, 0), neg_d = sum_g min(c_gd, 0)
//
// because max(c hi, c lo) = max(c, 0) hi + min(c, 0) lo for lo <= hi: the heads of a group meet in one pooled query, so
// a page costs 2 dim multiplications however many heads share it.  Pooled values have up to 13 bits and a sign; they are
// taken as lo + 128 hi with both in 8 bits, so that four products go into one instruction, and all sums are whole.
//
// A record of 2 dim bytes is read by as many lanes as it has 16-byte pieces (rounded up to a power of two); a lane keeps
// its piece of the pooled query in registers.  The k-th largest score is found by counting: the range of the scores is
// cut into 256 bins, the bin that holds the k-th becomes the range, at most four times; then one pass writes the blocks
// above it and the first of those equal to it, in ascending order.
//
// One workgroup per query and kv head does all of it while there are enough of those to fill the GPU or few blocks;
// otherwise the scores are made by workgroups of 64 blocks and pass through the workspace.
#include "tbn_kv.h"

namespace tbn {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWavesOf = kThreads / kWave;
constexpr int kInLds = 16384;     // scores of one query and kv head that are kept in LDS
constexpr int kSliced = 64;       // blocks of a workgroup that only scores

struct SelectArgs {
    tbn_kv_pool p;
    tbn_kv_index ix;
    KvQueries q;
    int32_t *picks;
    int32_t n_select, n_sink, n_recent;
    uint32_t *scores;   // (token, kv head, blocks) or NULL
    int32_t blocks;     // of the longest sequence
};

struct Pooled {
    float most[kWavesOf];
    __align__(16) int8_t lo[2 * kMaxDim], hi[2 * kMaxDim];
};

// Larger score, larger word.  Scores are never -0 or not a number.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t u = __float_as_uint(f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The pooled query of token `tok` and a kv head, in LDS.  Ends with a barrier.
template <typename T>
__device__ void pool_query(const SelectArgs &a, int64_t tok, int head, Pooled &l) {
    const int tid = threadIdx.x, D = a.p.dim, G = a.q.heads / a.p.kv_heads;
    const T *q = static_cast<const T *>(a.q.q) + tok * a.q.q_stride + int64_t(head) * G * D + tid;
    float most = 0.f;
    if (tid < D)
        for (int g = 0; g < G; ++g) {
            const float f = fabsf(ElemIO<T>::load(q + g * D));
            most = f < INFINITY ? fmaxf(most, f) : most;
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    if ((tid & 63) == 0) l.most[tid >> 6] = most;
    __syncthreads();
    const float up = pow2_of(6 - exponent_of(fmaxf(fmaxf(l.most[0], l.most[1]), fmaxf(l.most[2], l.most[3]))));
    if (tid < D) {
        int pos = 0, neg = 0;
        for (int g = 0; g < G; ++g) {
            const float f = ElemIO<T>::load(q + g * D);
            const int c = fabsf(f) < INFINITY ? static_cast<int>(rintf(f * up)) : 0;
            pos += max(c, 0);
            neg += min(c, 0);
        }
        l.lo[tid] = static_cast<int8_t>(pos % 128);
        l.hi[tid] = static_cast<int8_t>(pos / 128);
        l.lo[D + tid] = static_cast<int8_t>(neg % 128);
        l.hi[D + tid] = static_cast<int8_t>(neg / 128);
    }
    __syncthreads();
}

// Scores of blocks [from, to): put(block, word).  LANES: lanes per record.
template <int LANES, typename Put>
__device__ __forceinline__ void score_blocks(const SelectArgs &a, const int32_t *table, int head, int from, int to, const Pooled &l, Put put) {
    constexpr int kAt = kThreads / LANES, kDepth = 4;   // records at once, rounds in flight
    const int piece = threadIdx.x % LANES, mine = threadIdx.x / LANES, D = a.p.dim, KV = a.p.kv_heads;
    const bool there = piece * 16 < 2 * D;
    u32x4_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    if (there) {
        lo = *reinterpret_cast<const u32x4_t *>(l.lo + piece * 16);
        hi = *reinterpret_cast<const u32x4_t *>(l.hi + piece * 16);
    }
    for (int b0 = from + mine; b0 < to; b0 += kAt * kDepth) {
        int64_t record[kDepth];
        u32x4_t w[kDepth];
        float step[kDepth];
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            const int b = min(b0 + j * kAt, to - 1);
            record[j] = int64_t(page_in(table[b], static_cast<int>(a.p.n_pages))) * KV + head;
        }
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            w[j] = u32x4_t{0, 0, 0, 0};
            if (there) w[j] = *reinterpret_cast<const u32x4_t *>(a.p.summary + record[j] * (2 * D) + piece * 16);
            step[j] = a.p.step[record[j]];
        }
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            int s0 = 0, s1 = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s0 = __builtin_amdgcn_sdot4(static_cast<int>(w[j][e]), static_cast<int>(lo[e]), s0, false);
                s1 = __builtin_amdgcn_sdot4(static_cast<int>(w[j][e]), static_cast<int>(hi[e]), s1, false);
            }
            int sum = s0 + 128 * s1;
#pragma unroll
            for (int d = LANES / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
            const int b = b0 + j * kAt;
            if (piece == 0 && b < to) put(b, ordered(step[j] < INFINITY ? static_cast<float>(sum) * step[j] : INFINITY));
        }
    }
}

template <typename Put>
__device__ __forceinline__ void score_blocks(const SelectArgs &a, const int32_t *table, int head, int from, int to, const Pooled &l, Put put) {
    if (a.p.dim <= 64) score_blocks<8>(a, table, head, from, to, l, put);
    else if (a.p.dim <= 128) score_blocks<16>(a, table, head, from, to, l, put);
    else score_blocks<32>(a, table, head, from, to, l, put);
}

// A token's sequence, its own block and the blocks that are scored: [lo, hi).
struct Query {
    int64_t tok;
    int last, lo, hi;
    const int32_t *table;
    bool there;
};

__device__ __forceinline__ Query query_of(const SelectArgs &a, int s, int t) {
    Query r;
    const int t0 = max(a.q.cu_q[s], 0), T = min(a.q.cu_q[s + 1], static_cast<int>(a.q.total_q)) - t0;
    const int len = len_in(a.ix.lens[s], a.q.max_len), shift = __ffs(a.p.page) - 1;
    r.there = t < min(T, a.q.max_q);
    r.tok = t0 + t;
    const int own = min(max(len - T, 0) + t, len - 1);   // -1: an empty sequence
    r.last = own < 0 ? -1 : own >> shift;
    const bool all = r.last + 1 <= a.n_select;
    r.lo = all ? 0 : a.n_sink;
    r.hi = all ? 0 : r.last - a.n_recent + 1;
    r.table = a.ix.table + int64_t(s) * a.ix.max_pages;
    return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_score_kernel(SelectArgs a) {
    __shared__ Pooled pooled;
    const int slices = (a.blocks + kSliced - 1) / kSliced, slice = blockIdx.x % slices, t = blockIdx.x / slices, head = blockIdx.y;
    const Query r = query_of(a, blockIdx.z, t);
    const int from = max(r.lo, slice * kSliced), to = min(r.hi, (slice + 1) * kSliced);
    if (!r.there || from >= to) return;
    pool_query<T>(a, r.tok, head, pooled);
    uint32_t *out = a.scores + (r.tok * a.p.kv_heads + head) * a.blocks;
    score_blocks(a, r.table, head, from, to, pooled, [&](int b, uint32_t word) { out[b] = word; });
}

struct SelectLds {
    uint32_t bins[kThreads];
    uint32_t least[kWavesOf], most[kWavesOf];
    uint32_t part[2][kWavesOf];
    uint32_t bin, above;
    bool all;
};

// inclusive prefix over the workgroup's threads; ends with the totals of the waves read by everyone
__device__ __forceinline__ uint32_t prefix(uint32_t v, uint32_t *part, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) {
        before += w < wave ? part[w] : 0u;
        total += part[w];
    }
    return before + sum;
}

// SCORED: the scores are in a.scores; IN_LDS: they are (or come) into LDS.
template <typename T, bool SCORED, bool IN_LDS>
__global__ __launch_bounds__(kThreads) void kv_select_kernel(SelectArgs a) {
    extern __shared__ uint32_t kept[];
    __shared__ Pooled pooled;
    __shared__ SelectLds l;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, head = blockIdx.y;
    const Query r = query_of(a, blockIdx.z, blockIdx.x);
    if (!r.there) return;
    const int64_t row = r.tok * a.p.kv_heads + head;
    int32_t *picks = a.picks + row * a.n_select;
    if (r.hi <= r.lo) {   // no choice
        for (int i = tid; i < a.n_select; i += kThreads) picks[i] = i <= r.last ? i : -1;
        return;
    }
    const int n = r.hi - r.lo;
    const uint32_t k = a.n_select - a.n_sink - a.n_recent;   // at most n - 1: there are more blocks than picks
    for (int i = tid; i < a.n_sink; i += kThreads) picks[i] = i;
    for (int i = tid; i < a.n_recent; i += kThreads) picks[a.n_select - a.n_recent + i] = r.hi + i;
    if (k == 0) return;
    const uint32_t *scored = SCORED ? a.scores + row * a.blocks + r.lo : nullptr;
    if constexpr (!SCORED) {
        pool_query<T>(a, r.tok, head, pooled);
        score_blocks(a, r.table, head, r.lo, r.hi, pooled, [&](int b, uint32_t word) { kept[b - r.lo] = word; });
        __syncthreads();
    } else if constexpr (IN_LDS) {
        for (int i = tid; i < n; i += kThreads) kept[i] = scored[i];
        __syncthreads();
    }
    const uint32_t *words = IN_LDS ? kept : scored;

    uint32_t least = 0xffffffffu, most = 0;
    for (int i = tid; i < n; i += kThreads) {
        least = min(least, words[i]);
        most = max(most, words[i]);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        least = min(least, static_cast<uint32_t>(__shfl_xor(static_cast<int>(least), d)));
        most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), d)));
    }
    if (lane == 0) {
        l.least[wave] = least;
        l.most[wave] = most;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) {
        least = min(least, l.least[w]);
        most = max(most, l.most[w]);
    }
    uint32_t above = 0;   // words beyond `most`
    while (least < most) {   // the k-th largest word is in [least, most]
        const int cut = max(24 - __clz(most - least), 0);   // (most - least) >> cut is below 256
        l.bins[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const uint32_t w = words[i];
            if (w >= least && w <= most) atomicAdd(&l.bins[(w - least) >> cut], 1u);
        }
        __syncthreads();
        const uint32_t here = l.bins[kThreads - 1 - tid];   // thread 0 has the highest bin
        uint32_t total;
        const uint32_t upto = above + prefix(here, l.part[0], total);
        if (upto >= k && upto - here < k) {   // exactly one thread
            l.bin = kThreads - 1 - tid;
            l.above = upto - here;
            l.all = upto == k;
        }
        __syncthreads();
        above = l.above;
        least += l.bin << cut;
        most = most - least < (1u << cut) ? most : least + ((1u << cut) - 1u);
        if (l.all) {   // the whole bin is taken: everything beyond the word in front of it (scores' words are above 0)
            most = --least;
            above = k;
        }
        __syncthreads();
    }
    // `least` is the k-th largest word; k - above of those equal to it are taken, the lowest blocks first
    const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint32_t more = 0, same = 0;
    for (int i = i0; i < i1; ++i) {
        more += words[i] > least;
        same += words[i] == least;
    }
    uint32_t total;
    uint32_t more_at = prefix(more, l.part[0], total) - more, same_at = prefix(same, l.part[1], total) - same;
    const uint32_t take = k - above;
    for (int i = i0; i < i1; ++i) {
        const uint32_t w = words[i];
        if (w > least || (w == least && same_at < take)) picks[a.n_sink + more_at + min(same_at, take)] = r.lo + i;
        more_at += w > least;
        same_at += w == least;
    }
}

// The scores pass through the workspace where the queries and heads alone leave CUs idle and there is enough to share out, or
// where they do not fit into LDS.
bool sliced(const tbn_kv_pool &p, const KvQueries &q, int64_t blocks) {
    return blocks > kInLds || (q.total_q * p.kv_heads < 128 && blocks > 512);
}

int64_t blocks_of(const tbn_kv_pool &p, const KvQueries &q) { return (q.max_len + p.page - 1) / p.page; }

template <typename T>
tbn_status launch_select_typed(const SelectArgs &a, bool split, hipStream_t stream) {
    const dim3 grid(a.q.max_q, a.p.kv_heads, a.ix.n_seqs), block(kThreads);
    const unsigned lds = a.blocks <= kInLds ? 4u * a.blocks : 0u;
    if (split) {
        const int64_t slices = (a.blocks + kSliced - 1) / kSliced;
        if (slices * a.q.max_q > 0x7fffffffLL) {
            set_error("tbn_block_select: %d queries of %lld slices are beyond one launch", a.q.max_q, (long long)slices);
            return TBN_ERR_UNSUPPORTED;
        }
        hipLaunchKernelGGL((kv_score_kernel<T>), dim3(static_cast<unsigned>(slices * a.q.max_q), a.p.kv_heads, a.ix.n_seqs), block, 0, stream, a);
        if (lds) hipLaunchKernelGGL((kv_select_kernel<T, true, true>), grid, block, lds, stream, a);
        else hipLaunchKernelGGL((kv_select_kernel<T, true, false>), grid, block, 0, stream, a);
    } else {
        hipLaunchKernelGGL((kv_select_kernel<T, false, true>), grid, block, lds, stream, a);
    }
    return check_launch("tbn_block_select");
}

template <typename T>
hipError_t allow_lds() {   // 64 KiB of scores and the static arrays
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_select_kernel<T, true, true>), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * kInLds);
    return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_select_kernel<T, false, true>), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * kInLds);
}

}  // namespace

size_t block_select_workspace(const tbn_kv_pool &p, const tbn_kv_index &, const KvQueries &q) {
    const int64_t blocks = blocks_of(p, q);
    return sliced(p, q, blocks) ? static_cast<size_t>(q.total_q) * p.kv_heads * blocks * 4 : 0;
}

tbn_status launch_block_select(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t *picks, int32_t n_select, int32_t n_sink,
                               int32_t n_recent, uint32_t *ws, hipStream_t stream) {
    static const hipError_t attr = [] {
        const hipError_t e = allow_lds<float>();
        return e != hipSuccess ? e : allow_lds<uint16_t>();
    }();
    if (attr != hipSuccess) {
        set_error("tbn_block_select: %s", hipGetErrorString(attr));
        return TBN_ERR_DEVICE;
    }
    const int64_t blocks = blocks_of(p, q);
    const SelectArgs a{p, ix, q, picks, n_select, n_sink, n_recent, ws, static_cast<int32_t>(blocks)};
    const bool split = sliced(p, q, blocks);
    return p.dt == TBN_F32 ? launch_select_typed<float>(a, split, stream) : launch_select_typed<uint16_t>(a, split, stream);
}

}  // namespace tbn
