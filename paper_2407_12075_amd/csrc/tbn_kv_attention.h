// What the attention kernels share (tbn_kv_attention.hip, tbn_kv_rows.hip): arguments, operands, masks.
#pragma once
#include <cfloat>

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

struct AttentionArgs {   // of one launch
    tbn_kv_pool p;
    tbn_kv_index ix;
    KvQueries q;
    void *out;
    float *lse;
    const uint32_t *mask;
    int32_t mask_words;
    const int32_t *picks;
    int32_t n_select;
    float c;            // |scale| log2 e, never 0 (times an infinite logit it would be no number)
    uint32_t flip;      // sign bits of the query's elements, where the scale is negative
    float *part_o;      // (chunk, token, head, dim) sums, where the keys are split
    float4 *part_ml;    // (chunk, token, head) reference, sum of the weights, sum of the rounded weights, -
    int32_t chunk;      // keys, or picks, of a workgroup
    int32_t n_chunks;
    int32_t row_tiles;  // tiles of a workgroup's rows
};

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
    v.t0 = max(a.q.cu_q[s], 0);
    const int all = min(a.q.cu_q[s + 1], static_cast<int>(a.q.total_q)) - v.t0;
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

// picked blocks, bfloat16: queries that share a workgroup (0: none), 32 rows at most
int picked_queries(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_select);
void launch_kv_picked(const AttentionArgs &a, int queries, dim3 grid, hipStream_t stream);
// many rows, bfloat16: `tiles` (2 or 4) of 32 rows per workgroup
void launch_kv_rows(const AttentionArgs &a, int tiles, bool tokens, dim3 grid, hipStream_t stream);

}  // namespace tbn
