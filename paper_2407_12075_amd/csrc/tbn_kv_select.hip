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
// cut into 256 bins, the bin that holds the k-th becomes the range, at most four times and until it holds only scores that
// are taken; then one pass writes the blocks above it and the first of those equal to it, in ascending order.  The scores
// stay in registers, ranks come from ballots and sums over lanes from data-parallel moves: what costs time here are the
// barriers (one per cut).
//
// One workgroup per query and kv head does all of it while there are enough of those to fill the GPU or few blocks;
// otherwise the scores are made by workgroups of 64 blocks and pass through the workspace.
#include "tbn_kv.h"

namespace tbn {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWavesOf = kThreads / kWave;
constexpr int kInLds = 16384;     // scores of one query and kv head that a workgroup keeps (64 of a thread)
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

// The largest over the lanes of a wave, in the same way as prefix_of_lanes.
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t v) {   // in lane 63, for all
    v = max(v, from_lane<0x111, 0xf>(v));
    v = max(v, from_lane<0x112, 0xf>(v));
    v = max(v, from_lane<0x114, 0xf>(v));
    v = max(v, from_lane<0x118, 0xf>(v));
    v = max(v, from_lane<0x142, 0xa>(v));
    v = max(v, from_lane<0x143, 0xc>(v));
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}

// sum over neighbouring LANES lanes, in all of them
template <int LANES>
__device__ __forceinline__ int sum_of_lanes(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, false);    // one lane on within pairs, two within fours,
    v += __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);   // mirrored within eight, within sixteen
    if (LANES > 8) v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);
    if (LANES > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = static_cast<int>(r[0] + r[1]);
    }
    return v;
}

// The pooled query of token `tok` and a kv head, in LDS.  Ends with a barrier.
template <typename T>
__device__ void pool_query(const SelectArgs &a, int64_t tok, int head, Pooled &l) {
    const int tid = threadIdx.x, D = a.p.dim, G = a.q.heads / a.p.kv_heads;
    const T *q = static_cast<const T *>(a.q.q) + tok * a.q.q_stride + int64_t(head) * G * D + tid;
    constexpr int kFirst = 8;   // heads that are kept between the two passes
    float kept[kFirst], most = 0.f;
    if (tid < D) {
#pragma unroll
        for (int g = 0; g < kFirst; ++g) kept[g] = g < G ? ElemIO<T>::load(q + g * D) : 0.f;
#pragma unroll
        for (int g = 0; g < kFirst; ++g) most = fabsf(kept[g]) < INFINITY ? fmaxf(most, fabsf(kept[g])) : most;
        for (int g = kFirst; g < G; ++g) {
            const float f = fabsf(ElemIO<T>::load(q + g * D));
            most = f < INFINITY ? fmaxf(most, f) : most;
        }
    }
    const uint32_t top = most_of_lanes(__float_as_uint(most));   // magnitudes order as their bits
    if ((tid & 63) == 0) l.most[tid >> 6] = __uint_as_float(top);
    __syncthreads();
    const float up = pow2_of(6 - exponent_of(fmaxf(fmaxf(l.most[0], l.most[1]), fmaxf(l.most[2], l.most[3]))));
    if (tid < D) {
        int pos = 0, neg = 0;
#pragma unroll
        for (int g = 0; g < kFirst; ++g) {
            const int c = fabsf(kept[g]) < INFINITY ? static_cast<int>(rintf(kept[g] * up)) : 0;
            pos += max(c, 0);
            neg += min(c, 0);
        }
        for (int g = kFirst; g < G; ++g) {
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

// Scores of blocks [from, to), whose pages are page_of(block): put(block, word).  LANES: lanes per record.
template <int LANES, int kDepth, typename Page, typename Put>
__device__ __forceinline__ void score_blocks(const SelectArgs &a, int head, int from, int to, const Pooled &l, Page page_of, Put put) {
    constexpr int kAt = kThreads / LANES;   // records at once; kDepth rounds in flight
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
            record[j] = int64_t(page_in(page_of(b), static_cast<int>(a.p.n_pages))) * KV + head;
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
            const int sum = sum_of_lanes<LANES>(s0 + 128 * s1);
            const int b = b0 + j * kAt;
            if (piece == 0 && b < to) put(b, ordered(step[j] < INFINITY ? static_cast<float>(sum) * step[j] : INFINITY));
        }
    }
}

template <int kDepth, typename Page, typename Put>
__device__ __forceinline__ void score_blocks(const SelectArgs &a, int head, int from, int to, const Pooled &l, Page page_of, Put put) {
    if (a.p.dim <= 64) score_blocks<8, kDepth>(a, head, from, to, l, page_of, put);
    else if (a.p.dim <= 128) score_blocks<16, kDepth>(a, head, from, to, l, page_of, put);
    else score_blocks<32, kDepth>(a, head, from, to, l, page_of, put);
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
    score_blocks<4>(a, head, from, to, pooled, [&](int b) { return r.table[b]; }, [&](int b, uint32_t word) { out[b] = word; });
}

struct SelectLds {
    uint32_t bins[3][kThreads];   // one that is filled, one that may still be read, one that is cleared for the next turn
    uint32_t least[kWavesOf], most[kWavesOf];
    uint2 counts[64 * kWavesOf];   // of a round's words in a wave: larger ones, equal ones
};

// SCORED: the scores are in a.scores.  NW: words of a thread, kept in registers; 0: any number, read again each time (SCORED only).
template <typename T, bool SCORED, int NW>
__global__ __launch_bounds__(kThreads) void kv_select_kernel(SelectArgs a) {
    extern __shared__ uint32_t made[];
    __shared__ Pooled pooled;
    __shared__ SelectLds l;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), head = blockIdx.y;
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
    l.bins[0][tid] = 0;
    const uint32_t *words = SCORED ? a.scores + row * a.blocks + r.lo : made;
    if constexpr (!SCORED) {
        // a block's page number lies where its score will, so that records do not wait for the table one by one
        for (int i = tid; i < n; i += kThreads) made[i] = r.table[r.lo + i];
        pool_query<T>(a, r.tok, head, pooled);   // ends with a barrier
        score_blocks<8>(a, head, r.lo, r.hi, pooled, [&](int b) { return static_cast<int32_t>(made[b - r.lo]); }, [&](int b, uint32_t word) { made[b - r.lo] = word; });
        __syncthreads();
    }
    // a thread's words are kThreads apart; 0 (less than any score's word) behind the last one
    uint32_t kept[NW > 0 ? NW : 1];
    if constexpr (NW > 0) {
#pragma unroll
        for (int j = 0; j < NW; ++j) kept[j] = j * kThreads + tid < n ? words[j * kThreads + tid] : 0u;
    }
    const int rounds = (n + kThreads - 1) / kThreads;
    auto each = [&](auto use) __attribute__((always_inline)) {   // use(round, word)
        if constexpr (NW > 0) {
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (NW <= 4 || j < rounds) use(j, kept[j]);
        } else {
            for (int j = 0; j < rounds; ++j) use(j, j * kThreads + tid < n ? words[j * kThreads + tid] : 0u);
        }
    };

    uint32_t least = 0xffffffffu, most = 0;
    each([&](int, uint32_t w) {
        least = min(least, w ? w : 0xffffffffu);
        most = max(most, w);
    });
    least = ~most_of_lanes(~least);
    most = most_of_lanes(most);
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
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    uint32_t above = 0;   // words beyond `most`
    for (int turn = 0; least < most; turn = turn == 2 ? 0 : turn + 1) {   // the k-th largest word is in [least, most]
        const int cut = max(24 - __clz(most - least), 0);   // (most - least) >> cut is below 256
        l.bins[turn == 2 ? 0 : turn + 1][tid] = 0;
        each([&](int, uint32_t w) {
            if (w >= least && w <= most) atomicAdd(&l.bins[turn][(w - least) >> cut], 1u);
        });
        __syncthreads();
        // every wave finds the bin by itself: lane 0 has the four highest ones
        const uint4 b = *reinterpret_cast<const uint4 *>(&l.bins[turn][(kWave - 1 - lane) * 4]);
        const uint32_t here = b.x + b.y + b.z + b.w, upto = above + prefix_of_lanes(here);
        const int at = __ffsll(static_cast<long long>(__ballot(upto >= k))) - 1;   // the first lane that reaches k
        uint32_t sum = __builtin_amdgcn_readlane(upto - here, at);
        const uint32_t four[4] = {static_cast<uint32_t>(__builtin_amdgcn_readlane(b.w, at)), static_cast<uint32_t>(__builtin_amdgcn_readlane(b.z, at)),
                                  static_cast<uint32_t>(__builtin_amdgcn_readlane(b.y, at)), static_cast<uint32_t>(__builtin_amdgcn_readlane(b.x, at))};
        int bin = (kWave - 1 - at) * 4 + 3, inside = four[0];
#pragma unroll
        for (int j = 1; j < 4; ++j)
            if (sum + inside < k) {
                sum += inside;
                inside = four[j];
                --bin;
            }
        above = sum;
        least += static_cast<uint32_t>(bin) << cut;
        most = most - least < (1u << cut) ? most : least + ((1u << cut) - 1u);
        if (sum + inside == k) {   // the whole bin is taken: everything beyond the word in front of it (scores' words are above 0)
            most = --least;
            above = k;
        }
    }
    // `least` is the k-th largest word; k - above of those equal to it are taken, the lowest blocks first
    const uint32_t take = k - above;
    auto write = [&](int j, uint32_t w, uint32_t more_before, uint32_t same_before) {
        const uint64_t more = __ballot(w > least), same = __ballot(w == least), below = (uint64_t(1) << lane) - 1;
        const uint32_t more_at = more_before + __popcll(more & below), same_at = same_before + __popcll(same & below);
        if (w > least || (w == least && same_at < take)) picks[a.n_sink + more_at + min(same_at, take)] = r.lo + j * kThreads + tid;
    };
    if constexpr (NW > 0) {
        each([&](int j, uint32_t w) {
            const uint64_t more = __ballot(w > least), same = __ballot(w == least);
            if (lane == 0) l.counts[j * kWavesOf + wave] = make_uint2(__popcll(more), __popcll(same));
        });
        __syncthreads();
        uint32_t more = 0, same = 0;
        each([&](int j, uint32_t w) {
            uint32_t more_at = more, same_at = same;
#pragma unroll
            for (int u = 0; u < kWavesOf; ++u) {
                const uint2 c = l.counts[j * kWavesOf + u];
                if (u < wave) more_at += c.x, same_at += c.y;
                more += c.x;
                same += c.y;
            }
            write(j, w, more_at, same_at);
        });
    } else {
        uint32_t more = 0, same = 0;
        for (int j = 0; j < rounds; ++j) {
            const uint32_t w = j * kThreads + tid < n ? words[j * kThreads + tid] : 0u;
            const uint64_t m = __ballot(w > least), e = __ballot(w == least);
            uint2 *counts = l.counts + (j & 1) * kWavesOf;   // the round before last has been read by everyone
            if (lane == 0) counts[wave] = make_uint2(__popcll(m), __popcll(e));
            __syncthreads();
            uint32_t more_at = more, same_at = same;
#pragma unroll
            for (int u = 0; u < kWavesOf; ++u) {
                const uint2 c = counts[u];
                if (u < wave) more_at += c.x, same_at += c.y;
                more += c.x;
                same += c.y;
            }
            write(j, w, more_at, same_at);
        }
    }
}

// ---- several queries of a sequence -------------------------------------------------------------------------------------------
//
// Eight neighbouring queries share a workgroup and a read of each record: the scores are a matrix product of the records (rows) and
// the pooled queries' two bytes per channel (16 columns) on v_mfma_i32_16x16x64_i8.  A wave then picks for two of the queries by itself,
// without barriers.

typedef int i32x4_t __attribute__((ext_vector_type(4)));

constexpr int kQueries = 8;
constexpr int kTileBlocks = 2048;   // blocks of a sequence, at most (32 scores of a lane)

// Picks of one query by one wave: the k largest of words[0, n), block r0 + i for word i, in ascending order to picks.  NW * 64 >= n.
template <int NW>
__device__ __forceinline__ void pick_by_wave(const uint32_t *words, int n, uint32_t k, uint32_t *bins, int r0, int32_t *picks) {
    const int lane = threadIdx.x & 63;
    uint32_t kept[NW], least = 0xffffffffu, most = 0;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        kept[j] = j * kWave + lane < n ? words[j * kWave + lane] : 0u;
        least = min(least, kept[j] ? kept[j] : 0xffffffffu);
        most = max(most, kept[j]);
    }
    least = ~most_of_lanes(~least);
    most = most_of_lanes(most);
    uint32_t above = 0;
    while (least < most) {   // as in kv_select_kernel
        const int cut = max(24 - __clz(most - least), 0);
        *reinterpret_cast<uint4 *>(bins + lane * 4) = make_uint4(0, 0, 0, 0);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < NW; ++j)
            if (kept[j] >= least && kept[j] <= most) atomicAdd(&bins[(kept[j] - least) >> cut], 1u);
        __builtin_amdgcn_wave_barrier();
        const uint4 b = *reinterpret_cast<const uint4 *>(bins + (kWave - 1 - lane) * 4);
        __builtin_amdgcn_wave_barrier();
        const uint32_t here = b.x + b.y + b.z + b.w, upto = above + prefix_of_lanes(here);
        const int at = __ffsll(static_cast<long long>(__ballot(upto >= k))) - 1;
        uint32_t sum = __builtin_amdgcn_readlane(upto - here, at), inside = __builtin_amdgcn_readlane(b.w, at);
        const uint32_t rest[3] = {static_cast<uint32_t>(__builtin_amdgcn_readlane(b.z, at)), static_cast<uint32_t>(__builtin_amdgcn_readlane(b.y, at)),
                                  static_cast<uint32_t>(__builtin_amdgcn_readlane(b.x, at))};
        int bin = (kWave - 1 - at) * 4 + 3;
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (sum + inside < k) {
                sum += inside;
                inside = rest[j];
                --bin;
            }
        above = sum;
        least += static_cast<uint32_t>(bin) << cut;
        most = most - least < (1u << cut) ? most : least + ((1u << cut) - 1u);
        if (sum + inside == k) {
            most = --least;
            above = k;
        }
    }
    const uint32_t take = k - above;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    uint32_t more_at = 0, same_at = 0;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        const uint64_t more = __ballot(kept[j] > least), same = __ballot(kept[j] == least);
        const uint32_t m = more_at + __popcll(more & below), e = same_at + __popcll(same & below);
        if (kept[j] > least || (kept[j] == least && e < take)) picks[m + min(e, take)] = r0 + j * kWave + lane;
        more_at += __popcll(more);
        same_at += __popcll(same);
    }
}

// PRODUCTS: of 64 bytes of a record each
template <typename T, int PRODUCTS>
__global__ __launch_bounds__(kThreads, 4) void kv_select_tile_kernel(SelectArgs a) {
    extern __shared__ uint32_t words[];                                 // kQueries x blocks
    __shared__ __align__(16) int8_t pooled[2 * kQueries][2 * kMaxDim];   // columns: the low bytes of the queries, the high ones
    __shared__ __align__(16) uint32_t bins[kWavesOf][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int head = blockIdx.y, t_first = blockIdx.x * kQueries, D = a.p.dim, KV = a.p.kv_heads, G = a.q.heads / KV;
    const Query first = query_of(a, blockIdx.z, t_first);
    if (!first.there) return;
    int top = 0;   // blocks that some query of the tile scores: [n_sink, top)
#pragma unroll
    for (int t = 0; t < kQueries; ++t) {
        const Query r = query_of(a, blockIdx.z, t_first + t);
        if (r.there) top = max(top, r.hi);
    }
    const int lo = a.n_sink, count = top - lo;
    if (count > 0) {
        // pooled queries: a wave per query, lanes on channels
        for (int t = wave; t < kQueries; t += kWavesOf) {
            const Query r = query_of(a, blockIdx.z, t_first + t);
            float most = 0.f;
            const T *q = static_cast<const T *>(a.q.q) + (r.there ? r.tok : first.tok) * a.q.q_stride + int64_t(head) * G * D;
#pragma unroll 4
            for (int i = lane; i < G * D; i += kWave) {
                const float f = fabsf(ElemIO<T>::load(q + i));
                most = f < INFINITY ? fmaxf(most, f) : most;
            }
            const float up = pow2_of(6 - exponent_of(__uint_as_float(most_of_lanes(__float_as_uint(most)))));
            for (int d = lane; d < kMaxDim; d += kWave) {
                int pos = 0, neg = 0;
                if (d < D)
#pragma unroll 4
                    for (int u = 0; u < G; ++u) {
                        const float f = ElemIO<T>::load(q + u * D + d);
                        const int c = fabsf(f) < INFINITY ? static_cast<int>(rintf(f * up)) : 0;
                        pos += max(c, 0);
                        neg += min(c, 0);
                    }
                if (d < D) {
                    pooled[t][d] = static_cast<int8_t>(pos % 128);
                    pooled[kQueries + t][d] = static_cast<int8_t>(pos / 128);
                    pooled[t][D + d] = static_cast<int8_t>(neg % 128);
                    pooled[kQueries + t][D + d] = static_cast<int8_t>(neg / 128);
                }
            }
        }
        __syncthreads();
        i32x4_t column[PRODUCTS];
#pragma unroll
        for (int m = 0; m < PRODUCTS; ++m) {
            column[m] = i32x4_t{0, 0, 0, 0};
            if (64 * m + 16 * g < 2 * D) column[m] = *reinterpret_cast<const i32x4_t *>(&pooled[n][64 * m + 16 * g]);
        }
        for (int b0 = wave * 16; b0 < count; b0 += kWavesOf * 16) {
            const int64_t mine = int64_t(page_in(first.table[lo + min(b0 + n, count - 1)], static_cast<int>(a.p.n_pages))) * KV + head;
            const int8_t *record = a.p.summary + mine * (2 * D) + 16 * g;
            const float step = a.p.step[mine];   // of record n; rows come out four to a lane
            i32x4_t row[PRODUCTS], sum = {0, 0, 0, 0};
#pragma unroll
            for (int m = 0; m < PRODUCTS; ++m) {
                row[m] = i32x4_t{0, 0, 0, 0};
                if (64 * m + 16 * g < 2 * D) row[m] = *reinterpret_cast<const i32x4_t *>(record + 64 * m);
            }
#pragma unroll
            for (int m = 0; m < PRODUCTS; ++m)
                sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(row[m], column[m], sum, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int high = __builtin_amdgcn_update_dpp(0, sum[j], 0x128, 0xf, 0xf, false);   // eight lanes on in the row
                const int b = b0 + 4 * g + j;
                const float st = __shfl(step, 4 * g + j);
                if (n < kQueries && b < count)
                    words[n * a.blocks + b] = ordered(st < INFINITY ? static_cast<float>(sum[j] + 128 * high) * st : INFINITY);
            }
        }
        __syncthreads();
    }
    for (int t = wave; t < kQueries; t += kWavesOf) {
        const Query r = query_of(a, blockIdx.z, t_first + t);
        if (!r.there) break;
        int32_t *picks = a.picks + (r.tok * KV + head) * a.n_select;
        if (r.hi <= r.lo) {   // no choice
            for (int i = lane; i < a.n_select; i += kWave) picks[i] = i <= r.last ? i : -1;
            continue;
        }
        for (int i = lane; i < a.n_sink; i += kWave) picks[i] = i;
        for (int i = lane; i < a.n_recent; i += kWave) picks[a.n_select - a.n_recent + i] = r.hi + i;
        const uint32_t k = a.n_select - a.n_sink - a.n_recent, *mine = words + t * a.blocks;
        const int m = r.hi - r.lo;
        if (k == 0) continue;
        if (m <= 4 * kWave) pick_by_wave<4>(mine, m, k, bins[wave], r.lo, picks + a.n_sink);
        else if (m <= 12 * kWave) pick_by_wave<12>(mine, m, k, bins[wave], r.lo, picks + a.n_sink);
        else pick_by_wave<32>(mine, m, k, bins[wave], r.lo, picks + a.n_sink);
    }
}

bool tiled(const KvQueries &q, int64_t blocks) { return q.max_q > 1 && blocks <= kTileBlocks; }

// One query at a time: the scores pass through the workspace where the queries and heads alone leave CUs idle and there is enough to share out, or
// where they do not fit into LDS.
bool sliced(const tbn_kv_pool &p, const KvQueries &q, int64_t blocks) {
    return !tiled(q, blocks) && (blocks > kInLds || (q.total_q * p.kv_heads < 128 && blocks > 512));
}

int64_t blocks_of(const tbn_kv_pool &p, const KvQueries &q) { return (q.max_len + p.page - 1) / p.page; }

template <typename T, bool SCORED>
void launch_select_kernel(const SelectArgs &a, hipStream_t stream) {
    const dim3 grid(a.q.max_q, a.p.kv_heads, a.ix.n_seqs), block(kThreads);
    const unsigned lds = SCORED ? 0u : 4u * a.blocks;
    if (a.blocks <= 4 * kThreads) hipLaunchKernelGGL((kv_select_kernel<T, SCORED, 4>), grid, block, lds, stream, a);
    else if (a.blocks <= 16 * kThreads) hipLaunchKernelGGL((kv_select_kernel<T, SCORED, 16>), grid, block, lds, stream, a);
    else if (!SCORED || a.blocks <= kInLds) hipLaunchKernelGGL((kv_select_kernel<T, SCORED, 64>), grid, block, lds, stream, a);
    else hipLaunchKernelGGL((kv_select_kernel<T, true, 0>), grid, block, lds, stream, a);
}

template <typename T>
tbn_status launch_select_typed(const SelectArgs &a, bool split, hipStream_t stream) {
    if (tiled(a.q, a.blocks)) {
        const dim3 grid((a.q.max_q + kQueries - 1) / kQueries, a.p.kv_heads, a.ix.n_seqs);
        const unsigned lds = 4u * kQueries * a.blocks;
        if (a.p.dim <= 64) hipLaunchKernelGGL((kv_select_tile_kernel<T, 2>), grid, dim3(kThreads), lds, stream, a);
        else if (a.p.dim <= 128) hipLaunchKernelGGL((kv_select_tile_kernel<T, 4>), grid, dim3(kThreads), lds, stream, a);
        else hipLaunchKernelGGL((kv_select_tile_kernel<T, 8>), grid, dim3(kThreads), lds, stream, a);
    } else if (split) {
        const int64_t slices = (a.blocks + kSliced - 1) / kSliced;
        if (slices * a.q.max_q > 0x7fffffffLL) {
            set_error("tbn_block_select: %d queries of %lld slices are beyond one launch", a.q.max_q, (long long)slices);
            return TBN_ERR_UNSUPPORTED;
        }
        hipLaunchKernelGGL((kv_score_kernel<T>), dim3(static_cast<unsigned>(slices * a.q.max_q), a.p.kv_heads, a.ix.n_seqs), dim3(kThreads), 0, stream, a);
        launch_select_kernel<T, true>(a, stream);
    } else {
        launch_select_kernel<T, false>(a, stream);
    }
    return check_launch("tbn_block_select");
}

template <typename T>
hipError_t allow_lds() {   // up to 64 KiB of scores beside the static arrays
    const void *kernels[] = {reinterpret_cast<const void *>(&kv_select_kernel<T, false, 64>), reinterpret_cast<const void *>(&kv_select_tile_kernel<T, 2>),
                             reinterpret_cast<const void *>(&kv_select_tile_kernel<T, 4>), reinterpret_cast<const void *>(&kv_select_tile_kernel<T, 8>)};
    static_assert(kQueries * kTileBlocks == kInLds, "one limit");
    for (const void *k : kernels)
        if (const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, 4 * kInLds); e != hipSuccess) return e;
    return hipSuccess;
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
