// What the attention kernels share (tbn_kv_attention.hip, tbn_kv_rows.hip): arguments, operands, masks.
#pragma once
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "tbn_kv.h"

namespace tbn {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kAttnWaves = 4;
constexpr int kAttnThreads = kAttnWaves * kWave;
constexpr int kListed = 1024;   // pages of a workgroup's stretch of keys, at most
constexpr float kSlack = 8.f;   // a row's sums are scaled down when a logit passes their reference by more: weights stay below 2^8
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct WindowArgs {
    int32_t sink, size;   // the first keys, which every token sees, and how many up to its own place
};

struct AttentionArgs {   // of one launch; not above 248 bytes (256 and 276 cost a call on one token 0.2 - 0.3 us)
    tbn_kv_pool p;      // a cache in 4 bits: k and v its codes, summary and step its exponents, dt the queries' type
    tbn_kv_index ix;
    KvQueries q;
    void *out;
    float *lse;
    const uint32_t *mask;
    int32_t mask_words;
    union {
        const int32_t *picks;   // of a call on picked pages
        WindowArgs window;      // of a call with a window
    };
    int32_t n_select;
    float c;            // |scale| log2 e, never 0 (times an infinite logit it would be no number)
    uint32_t flip;      // sign bits of the query's elements, where the scale is negative
    float *part_o;      // (chunk, token, head, dim) sums, where the keys are split
    float4 *part_ml;    // (chunk, token, head) reference, sum of the weights, sum of the rounded weights, -
    int32_t chunk;      // keys, or picks, of a workgroup
    int32_t n_chunks;
    int32_t row_tiles;  // tiles of a workgroup's rows
};

// what the rows of a launch see: every key up to their own, the pages they picked, the first keys and a window
enum Kind { kAll, kPicked, kWindow };

template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
    static constexpr int kStep = 32, kOf = 8;   // keys of a step, of a lane
    static constexpr int kTiles = 2;            // tiles of 16 keys of a step, which share their query operand
    typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
    // 1.0 where the bit is set
    static __device__ __forceinline__ u32x4_t ones(uint32_t bits) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = ((bits >> (2 * e)) & 1u ? 0x3f80u : 0u) | ((bits >> (2 * e + 1)) & 1u ? 0x3f800000u : 0u);
        return w;
    }
    // the first n values, 0 in place of the others
    static __device__ __forceinline__ u32x4_t first_of(u32x4_t w, int n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] &= n > 2 * e + 1 ? ~0u : n > 2 * e ? 0xffffu : 0u;
        return w;
    }
    static __device__ __forceinline__ bool not_finite(u32x4_t w) {
        bool is = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) is |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
        return is;
    }
    static __device__ __forceinline__ u32x4_t finite_of(u32x4_t w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] &= ((w[e] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w[e] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
        return w;
    }
    // values with 0 for those that are not finite, and the kinds of those (limit_of)
    static __device__ __forceinline__ void part(u32x4_t w, u32x4_t &finite, u32x4_t &kinds) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t fin = 0, kin = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t x = (w[e] >> (16 * h)) & 0xffffu;
                if ((x & 0x7f80u) != 0x7f80u) fin |= x << (16 * h);
                else kin |= (x & 0x7fu ? 0x4580u : x & 0x8000u ? 0x4280u : 0x3f80u) << (16 * h);
            }
            finite[e] = fin;
            kinds[e] = kin;
        }
    }
};
template <> struct Elem<float> {
    static constexpr int kStep = 16, kOf = 4, kTiles = 1;
    typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ u32x4_t ones(uint32_t bits) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bits >> e) & 1u ? 0x3f800000u : 0u;
        return w;
    }
    static __device__ __forceinline__ u32x4_t first_of(u32x4_t w, int n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = n > e ? w[e] : 0u;
        return w;
    }
    static __device__ __forceinline__ bool not_finite(u32x4_t w) {
        bool is = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) is |= (w[e] & 0x7f800000u) == 0x7f800000u;
        return is;
    }
    static __device__ __forceinline__ u32x4_t finite_of(u32x4_t w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (w[e] & 0x7f800000u) == 0x7f800000u ? 0u : w[e];
        return w;
    }
    static __device__ __forceinline__ void part(u32x4_t w, u32x4_t &finite, u32x4_t &kinds) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = w[e];
            const bool fin = (x & 0x7f800000u) != 0x7f800000u;
            finite[e] = fin ? x : 0u;
            kinds[e] = fin ? 0u : x & 0x7fffffu ? 0x45800000u : x & 0x80000000u ? 0x42800000u : 0x3f800000u;
        }
    }
};

// What `counts` infinite values and not-a-numbers that a row sees add to its sum (kinds: 1 for +infinity, 64 for -infinity, 4096 for
// not a number, so that a step's up to 32 keys of each can be told apart).
__device__ __forceinline__ float limit_of(float counts) {
    const uint32_t c = static_cast<uint32_t>(counts);
    const bool plus = c & 63u, minus = (c >> 6) & 63u;
    return c >= 4096u || (plus && minus) ? NAN : plus ? INFINITY : minus ? -INFINITY : 0.f;
}

// rows of a sequence: tokens x heads of the group; where its keys end for a row tile
struct Span {
    int t0, T, len, prefix;   // first token of the call, tokens, keys, keys before those tokens
};

__device__ __forceinline__ Span span_of(const AttentionArgs &a, int s) {
    Span v;
    const int all = tokens_in(a.q.cu_q, s, a.q.total_q, v.t0);
    v.T = min(all, a.q.max_q);
    v.len = len_in(a.ix.lens[s], a.q.max_len);
    v.prefix = max(v.len - max(all, 0), 0);
    return v;
}

// The sequence of a workgroup, -1 if there is nothing to do.  An index with more sequences than the call has tokens has idle ones: there the
// launch may have a row of workgroups for each token (TOKENS), and that of a sequence's first token does its work.  Their sequence is the last one that
// begins at or before the token: 64 places are looked at in each round.  (Instances of their own: a branch would cost every launch 0.5 us.)
template <bool TOKENS>
__device__ __forceinline__ int sequence_of(const AttentionArgs &a) {
    const int row = blockIdx.y;
    if constexpr (!TOKENS) return row;
    const int lane = threadIdx.x & 63;
    int s = 0, n = a.ix.n_seqs + 1;   // it is among the n entries of cu_q from s on
    while (n > 1) {
        const int step = (n + kWave - 1) / kWave;
        const int before = static_cast<int>(__popcll(__ballot(lane * step < n && a.q.cu_q[s + min(lane * step, n - 1)] <= row)));
        const int skip = max(before - 1, 0) * step;   // below n
        s += skip;
        n = min(step, n - skip);
    }
    s = __builtin_amdgcn_readfirstlane(s);
    return s < a.ix.n_seqs && max(a.q.cu_q[s], 0) == row ? s : -1;
}

// A workgroup's share.  Heads vary fastest: neighbouring workgroups go to different XCDs, so every XCD gets the same mix of stretches (a
// stretch that only the longest sequences have would otherwise always fall to the same ones: 64 ragged sequences took 655 us in place of
// 468), and with 8 kv heads the row tiles of one head share an L2.
struct Block {
    int head, row_tile, chunk, token;   // token: of a call on picked blocks
};

__device__ __forceinline__ Block block_of(const AttentionArgs &a) {
    Block b;
    uint32_t x = blockIdx.x;
    b.head = x % a.p.kv_heads;
    x /= a.p.kv_heads;
    b.row_tile = x % a.row_tiles;
    x /= a.row_tiles;
    b.chunk = x % a.n_chunks;
    b.token = x / a.n_chunks;
    return b;
}

__device__ __forceinline__ int keys_end(const AttentionArgs &a, const Span &v, int last_row, int G) {
    return a.mask ? v.len : min(v.len, v.prefix + last_row / G + 1);
}

// The keys that the rows [row0, row1] of a call with a window can see, as pages without a gap: the pages of the first keys, then those
// from the first row's window on.  "Within" counts keys along them; `gap` keys are left out behind the first `head` of them.  No more than a plan has
// stretches for (window_keys): with a mask keys of tokens beyond max_q, which the caller says there are none of, are left out.
struct Within {
    int head, gap, end, low;   // keys of the first pages, keys left out, keys in all, the least key of the first row's window
    __device__ __forceinline__ int key(int x) const { return x < head ? x : x + gap; }
};

__device__ __forceinline__ Within within_of(const AttentionArgs &a, const Span &v, int row0, int row1, int G, int shift) {
    const int end = min(keys_end(a, v, row1, G), v.prefix + v.T), pages = (end + a.p.page - 1) >> shift;
    Within w;
    // with a mask a row's place is what it has above it, none at least
    w.low = max((a.mask ? v.prefix - 1 : v.prefix + row0 / G) - a.window.size + 1, 0);
    const int sink = (min(a.window.sink, end) + a.p.page - 1) >> shift, from = w.low >> shift;
    w.head = sink << shift;
    w.gap = from > sink && from < pages ? (from - sink) << shift : 0;
    w.end = from >= pages ? min(w.head, end) : end - w.gap;
    return w;
}

// The least key of a row's window: its place is its own key's, with a mask the number of the tokens it sees more than the keys before the call.
// (There max_q <= window, so a window never ends among the call's own tokens.)
__device__ __forceinline__ int window_of(const AttentionArgs &a, const Span &v, int place) {
    int at = v.prefix + place;
    if (a.mask) {
        const uint32_t *mask = a.mask + int64_t(v.t0 + place) * a.mask_words;
        at = v.prefix - 1;
        for (int w = 0; w * 32 < v.T; ++w) at += __popc(mask[w] & (v.T - w * 32 >= 32 ? ~0u : (1u << (v.T - w * 32)) - 1u));
    }
    return at - a.window.size + 1;
}

// no row's window begins behind this key
__device__ __forceinline__ int last_window(const AttentionArgs &a, const Span &v, int row1, int G) {
    return v.prefix + (a.mask ? v.T - 1 : row1 / G) - a.window.size + 1;
}

// a word with its first n bits set, as far as it has them
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// the larger of a lane's value and that of the lane 32 away (16 away)
__device__ __forceinline__ float max_over_32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A weight is rounded to 8 bits for the product with v, as the values it multiplies have.  The sum that divides the product takes the
// rounded ones, so that a row that one key dominates is not scaled by that key's rounding; lse has a sum of its own.  Relative error of the output against 64
// bits: 1.9e-3 - 2.3e-3; 1.7e-3 is its own rounding, which weights of 32 bits would leave at the price of a float32 product or of a second one.
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}
__device__ __forceinline__ float add_two_bf16(uint32_t pair, float sum) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), sum, false);
}

// 2^x: exact to one unit in the last place; results below 2^-126 are 0
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// What a row's logits are counted from.  Finite, so that a row that has seen nothing yet gives weights of 0 (-infinity less a finite number) and
// an infinite logit one of infinity (infinity less infinity would be no number): its sum, and so lse, is infinity then.
__device__ __forceinline__ float reference_of(float m) { return __builtin_amdgcn_fmed3f(m, -FLT_MAX, FLT_MAX); }

// Which of a lane's `n` keys from `k0` on a row sees, as bits: keys before `end` and, among the call's own tokens, those of the row's mask
// or up to its place.
template <bool PICKED>
__device__ __forceinline__ uint32_t seen_bits(const AttentionArgs &a, const Span &v, int k0, int end, int place) {
    uint32_t bits = first_bits(end - k0);
    if (PICKED) return bits;
    const int j0 = k0 - v.prefix;   // place among the call's tokens, negative for the keys before them
    if (!a.mask) return bits & first_bits(place + 1 - j0);
    const uint32_t *mask = a.mask + int64_t(v.t0 + place) * a.mask_words;
    const int at = j0 >> 5;
    const uint32_t lo = at < 0 ? ~0u : at < a.mask_words ? mask[at] : 0u, hi = at < -1 ? ~0u : at + 1 < a.mask_words ? mask[at + 1] : 0u;
    return bits & __funnelshift_r(lo, hi, j0 & 31);
}

// with a window that begins at key `low`
template <Kind KIND>
__device__ __forceinline__ uint32_t seen_within(const AttentionArgs &a, const Span &v, int k0, int end, int place, int low) {
    uint32_t bits = seen_bits<KIND == kPicked>(a, v, k0, end, place);
    if constexpr (KIND == kWindow) bits &= first_bits(a.window.sink - k0) | ~first_bits(low - k0);
    return bits;
}

// Four channels of a row from its sums: to the output, or to the parts of its stretch.  m in units of log2; l the weights' sum, z the
// rounded weights'.
template <typename T>
__device__ __forceinline__ void store_sums(const AttentionArgs &a, int chunk, int64_t at, int d, f32x4_t sum, float m, float l, float z) {
    const int D = a.p.dim;
    if (a.n_chunks > 1) {
        const int64_t pa = int64_t(chunk) * a.q.total_q * a.q.heads + at;
        *reinterpret_cast<f32x4_t *>(a.part_o + pa * D + d) = sum;
        if (d == 0) a.part_ml[pa] = make_float4(m, l, z, 0.f);
    } else {
        const float inv = z == 0.f ? 0.f : 1.f / z;
        T *out = static_cast<T *>(a.out) + at * D + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) ElemIO<T>::store(out + e, sum[e] * inv);
        if (d == 0 && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
}

// How a call is spread over workgroups.
struct Plan {
    int rows, chunk, n_chunks, row_tiles;   // rows of a workgroup; stretches of keys
    bool staged;                            // by a kernel that stages keys in LDS
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Whether a launch has a row of workgroups per token of the call instead of per place of the index (sequence_of): where no token is without work, or
// places are many more.
inline bool by_token(const tbn_kv_index &ix, const KvQueries &q) { return q.total_q < ix.n_seqs && (q.max_q == 1 || 16 * q.total_q <= ix.n_seqs); }

// Workgroups of a launch whose rows may mostly be idle, at most: 0.2 - 0.6 ns each where they end at once, small against the work.
inline double most_blocks(int64_t keys) { return std::min(150000., 16384. + 8. * keys); }

// An index has room for more sequences than are there, so keys are split by the sequences of the call: max_q tokens each would be the fewest; drafts are
// ragged, half of max_q and more in the mean, so twice that (16 trees of up to 26 tokens: 49 us, 58 with the fewest).  One token on 131000 keys in one of 64
// places: 101 us, 1065 split by places; a tree of 26: 124 and 1383.  But every place (or token, whose idle workgroups take five times as long) has its row
// of workgroups: beyond most_blocks they are split as if for twice as many sequences, and so on up to one for each row.
// keys: that a sequence of the call has for a row of workgroups to go through, at most.  plan(rows of a sequence, sequences x kv heads, keys).
template <typename F>
Plan plan_by_sequences(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int64_t keys, F plan) {
    const int64_t rows = int64_t(q.max_q) * (q.heads / p.kv_heads);
    const bool token = by_token(ix, q);
    const int64_t most = token ? q.total_q : ix.n_seqs;
    const double weight = most * (token && q.max_q > 1 ? 5. : 1.), join = double(q.max_q) * q.heads;
    int64_t sequences = std::min<int64_t>({ix.n_seqs, q.total_q, 2 * ceil_div(q.total_q, q.max_q)});
    for (;; sequences = std::min(most, 2 * sequences)) {
        const Plan pl = plan(rows, sequences * p.kv_heads, keys);
        const double blocks = double(pl.n_chunks) * pl.row_tiles * p.kv_heads + (pl.n_chunks > 16 ? join : pl.n_chunks > 1 ? join / 4 : 0.);
        if (sequences >= most || blocks * weight <= most_blocks(keys)) return pl;
    }
}

// Keys of a window up to which rows alone are spread over the places: 8 kv heads of 128 channels, 1024 tokens, in tiles of 64 and unsplit against 128 and in parts: window
// 4000 94 us, 98; 8000 167, 162 (700 tokens: 146, 164); 16000 315, 289.
constexpr int64_t kFewKeys = 10240;

// Whether the rows of a call with a window are taken in tiles of 64 although they are more.  Its keys are few, so rows are what fills the places: where tiles of
// 128 would leave half of them empty, and those of 64 give every CU one (8 kv heads of 128 channels, window 1024, 1024 tokens: 38 us, 51 in tiles of 128 with the
// keys in two parts; on the cache in 4 bits 43, 54).  With fewer rows the keys are split in any case (300 tokens, window 4096: 54 us, in tiles of 128 52; in 4 bits 63, 54).
inline bool rows_of_64(int64_t rows, int64_t groups, int64_t keys, int64_t places) {
    return keys <= kFewKeys && groups * ceil_div(rows, 128) <= places / 2 && groups * ceil_div(rows, 64) >= places / 2;
}

// Keys that a workgroup of `rows` rows at most goes through in a call with a window, at most: the first pages, the window of its first row and
// what its other rows add.
inline int64_t window_keys(const tbn_kv_pool &p, const KvQueries &q, int32_t n_sink, int32_t window, bool masked, int rows = 128) {
    const int64_t tokens = masked ? q.max_q : std::min<int64_t>(q.max_q, rows / (q.heads / p.kv_heads) + 2);
    return std::min(q.max_len, ceil_div(n_sink, p.page) * p.page + window + tokens + 2 * p.page);
}

inline size_t workspace_of(const tbn_kv_pool &p, const KvQueries &q, const Plan &pl) {
    return pl.n_chunks > 1 ? static_cast<size_t>(pl.n_chunks) * q.total_q * q.heads * (p.dim + 4) * 4 : 0;
}

// c and the sign of a call's scale
inline float factor_of(float scale) {
    const float c = fabsf(scale) * kLog2e;
    return c < 1e-37f ? 1e-37f : c;
}
inline uint32_t flip_of(const tbn_kv_pool &p, float scale) { return !(scale < 0.f) ? 0u : p.dt == TBN_F32 ? 0x80000000u : 0x80008000u; }

constexpr int64_t kMostBlocks = 0x7fffffff;   // workgroups of a sequence

// Fills in how `pl` splits the call and the grid of its launch; an error where one launch cannot hold it.
tbn_status spread(AttentionArgs &a, const Plan &pl, float *ws, Kind kind, const char *what, dim3 &grid, bool &tokens);
// the cache in 4 bits, many rows, bfloat16: `tiles` (2 or 4) of 32 rows per workgroup
void launch_kv4_rows(const AttentionArgs &a, Kind kind, int tiles, bool tokens, dim3 grid, hipStream_t stream);
// the second kernel of a split call
void launch_kv_join(const AttentionArgs &a, Kind kind, int tile_rows, bool tokens, unsigned groups, hipStream_t stream);

static_assert(sizeof(AttentionArgs) <= 248, "kernel arguments");

// picked blocks, bfloat16: queries that share a workgroup (0: none), 32 rows at most
int picked_queries(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_select);
void launch_kv_picked(const AttentionArgs &a, int queries, dim3 grid, hipStream_t stream);
// many rows, bfloat16: `tiles` (2 or 4) of 32 rows per workgroup
void launch_kv_rows(const AttentionArgs &a, Kind kind, int tiles, bool tokens, dim3 grid, hipStream_t stream);

}  // namespace tbn
