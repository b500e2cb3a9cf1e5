// Attention over the paged cache: the tokens of a drafted tree (or a prompt chunk, or one token) over all keys of their
// sequence, and one query at a time over the blocks it picked.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c a_j - m),  c = scale * log2 e,  m the running maximum of c a_j
//
// One pass over the keys.  A workgroup takes rows (pairs of a token and a query head that share one kv head) in tiles of
// 16 and a stretch of keys; its waves take steps of 32 keys (float32: 16) in turn and each keeps a softmax of its own,
// merged through LDS at the end.  Both products run with keys or channels as rows of the matrix instruction and query
// rows as its columns:
//
//   S^T = K Q^T  (lane l: query row l % 16, the keys E (l / 16) .. + E - 1 of the step, E = 8 or 4)
//   O^T += V^T P^T
//
// The rows of K are dealt to the instruction's rows so that what comes out of the first product is what the second one
// takes: the weights stay in the lane that made them, already in operand order, and a row's maximum needs two exchanges
// between lanes per step.  K and V go from memory straight to registers in 16-byte pieces (V lies transposed in the
// cache); nothing of them passes through LDS.  The next step's K is requested when the first product has used this
// step's, its V when the second has.
//
// Where there are few rows the keys are split over workgroups as well; a second kernel joins the parts.
//
// A key that a row does not see: its logit is replaced, not added to.  Its value is still multiplied by a weight of 0, so
// in steps that hold such keys values behind the last visible key are replaced by 0, and if another value of the step is
// infinite or not a number it is replaced by 0 too and a third product counts, for each row, the ones that it sees.
#include "tbn_kv.h"

namespace tbn {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kListed = 1024;   // pages of a workgroup's stretch of keys, at most
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttentionArgs {
    tbn_kv_pool p;
    tbn_kv_index ix;
    KvQueries q;
    void *out;
    float *lse;
    const uint32_t *mask;
    int32_t mask_words;
    const int32_t *picks;
    int32_t n_select;
    float c;            // scale * log2 e
    float *part_o;      // (chunk, token, head, dim) sums, where the keys are split
    float2 *part_ml;    // (chunk, token, head) maximum and sum
    int32_t chunk;      // keys, or picks, of a workgroup
    int32_t n_chunks;
    int32_t row_tiles;  // of 16 * RT rows
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

__device__ __forceinline__ int keys_end(const AttentionArgs &a, const Span &v, int last_row, int G) {
    return a.mask ? v.len : min(v.len, v.prefix + last_row / G + 1);
}

// a word with its first n bits set, as far as it has them
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// 2^x: exact to one unit in the last place; results below 2^-126 are 0
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// RT: row tiles of a workgroup.  DP: channels the registers hold (dim <= DP; EVEN: dim == DP).
template <typename T, int DP, int RT, bool PICKED, bool EVEN>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void kv_attention_kernel(AttentionArgs a) {
    using E = Elem<T>;
    constexpr int KS = E::kStep, OF = E::kOf, NF = DP / 16, NQ = NF / E::kTiles;
    __shared__ int2 listed[kListed];   // slot and page
    __shared__ float sums[kWaves][16][DP + 4];
    __shared__ float maxima[kWaves][16], totals[kWaves][16];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int head = blockIdx.y, s = blockIdx.z, H = a.q.heads, KV = a.p.kv_heads, G = H / KV, D = a.p.dim, P = a.p.page;
    const int shift = __ffs(P) - 1;
    const Span v = span_of(a, s);
    int x = blockIdx.x;
    const int chunk = x % a.n_chunks;
    x /= a.n_chunks;
    const int base = (x % a.row_tiles) * (16 * RT);
    const int only = x / a.row_tiles;   // PICKED: the token
    const int R = PICKED ? G : v.T * G;   // rows of the sequence (PICKED: of the token)
    if (base >= R || (PICKED && only >= v.T)) return;
    const int own = v.prefix + only;   // PICKED: the query's own key
    const int end = PICKED ? min(v.len, own + 1) : keys_end(a, v, min(base + 16 * RT, R) - 1, G);

    // the pages of this stretch
    const int32_t *table = a.ix.table + int64_t(s) * a.ix.max_pages;
    const int n_pages = static_cast<int>(a.p.n_pages);
    int entries;
    if (PICKED) {
        const int first = chunk * a.chunk;
        entries = min(a.n_select - first, a.chunk);
        const int32_t *picks = a.picks + (int64_t(v.t0 + only) * KV + head) * a.n_select + first;
        for (int i = tid; i < entries; i += kThreads) {
            const int b = picks[i];
            const bool in = b >= 0 && b < (end + P - 1) >> shift;
            listed[i] = make_int2(in ? b : -1, in ? page_in(table[b], n_pages) : 0);
        }
    } else {
        const int first = chunk * a.chunk;
        if (first >= end && chunk > 0) return;
        entries = (min(end, first + a.chunk) - first + P - 1) >> shift;
        for (int i = tid; i < entries; i += kThreads) {
            const int slot = (first >> shift) + i;
            listed[i] = make_int2(slot, page_in(table[slot], n_pages));
        }
    }

    // this lane's query rows: its token's place and the operand of the first product
    u32x4_t q[RT][NQ];
    int place[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = base + r * 16 + n;
        const int t = PICKED ? only : min(row, R - 1) / G;
        place[r] = t;
        const T *src = static_cast<const T *>(a.q.q) + (v.t0 + t) * a.q.q_stride + (head * G + (PICKED ? row : row - t * G)) * D;
#pragma unroll
        for (int f = 0; f < NQ; ++f) {
            const int d = f * (4 * OF) + OF * g;
            u32x4_t w = {0, 0, 0, 0};
            if (row < R && (EVEN || d < D)) w = *reinterpret_cast<const typename E::u32x4_any *>(src + d);
            q[r][f] = w;
        }
    }

    f32x4_t o[RT][NF];
    float m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f) o[r][f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const int64_t page_elems = int64_t(P) * D;
    const T *kp = static_cast<const T *>(a.p.k) + head * page_elems, *vp = static_cast<const T *>(a.p.v) + head * page_elems;
    const int sub_shift = shift - (KS == 32 ? 5 : 4);
    const int steps = entries << sub_shift;
    // piece f of K: bfloat16 tile f % 2, channels 32 (f / 2) + 8 g; row n of tile 0 / 1 is key 8 (n / 4) + n % 4 (+ 4)
    const int k_key = OF == 8 ? 8 * (n >> 2) + (n & 3) : n;
    auto load_k = [&](u32x4_t (&k)[NF], int page, int off) {
        const T *src = kp + int64_t(page) * (page_elems * KV);
        const int o0 = (off + k_key) * D + (OF == 8 ? 8 * g : 4 * g);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int d = OF == 8 ? (f / 2) * 32 : f * 16;
            const int o1 = o0 + d + (OF == 8 ? (f & 1) * 4 * D : 0);
            u32x4_t w = {0, 0, 0, 0};
            if (EVEN || d + OF * g < D) w = *reinterpret_cast<const u32x4_t *>(src + o1);
            k[f] = w;
        }
    };
    auto load_v = [&](u32x4_t (&w)[NF], int page, int off) {
        const T *src = vp + int64_t(page) * (page_elems * KV);
        const int o0 = n * P + off + OF * g;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            u32x4_t x = {0, 0, 0, 0};
            if (EVEN || f * 16 + n < D) x = *reinterpret_cast<const u32x4_t *>(src + o0 + f * 16 * P);
            w[f] = x;
        }
    };
    // step i of this stretch: its first key, -1 if there is nothing in it; wave-uniform
    auto key_of = [&](int i, int &page) {
        const int2 e = listed[i >> sub_shift];
        page = __builtin_amdgcn_readfirstlane(e.y);
        const int slot = __builtin_amdgcn_readfirstlane(e.x);
        const int key = (slot << shift) + (i & ((1 << sub_shift) - 1)) * KS;
        return slot < 0 || key >= end ? -1 : key;
    };
    auto next_step = [&](int i, int &key, int &page) {
        while (i < steps) {
            key = key_of(i, page);
            if (key >= 0) break;
            i += kWaves;
        }
        return i;
    };

    __syncthreads();
    u32x4_t k[NF], w[NF];
    int key = 0, page = 0;
    int i = next_step(wave, key, page);
    if (i < steps) {
        load_k(k, page, key & (P - 1));
        load_v(w, page, key & (P - 1));
    }
    // keys from here on are not seen by every row
    const int all_see = PICKED ? end : a.mask ? v.prefix : v.prefix + base / G + 1;
    while (i < steps) {
        int next_key = 0, next_page = 0;
        const int next = next_step(i + kWaves, next_key, next_page);
        float p[RT][OF];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
            if constexpr (OF == 8) {
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    s0 = E::mma(k[f], q[r][f / 2], s0);
                    s1 = E::mma(k[f + 1], q[r][f / 2], s1);
                }
            } else {
#pragma unroll
                for (int f = 0; f < NF; ++f) s0 = E::mma(k[f], q[r][f], s0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[r][e] = s0[e] * a.c;
                if constexpr (OF == 8) p[r][4 + e] = s1[e] * a.c;
            }
        }
        if (next < steps) load_k(k, next_page, next_key & (P - 1));

        const bool edge = key + KS > all_see;   // wave-uniform
        uint32_t seen[RT];
        bool odd = false;
        if (edge) {
            const int k0 = key + OF * g;   // this lane's keys
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                uint32_t bits = first_bits(end - k0);
                if (!PICKED) {
                    const int j0 = k0 - v.prefix;   // place among the call's tokens, negative for the keys before them
                    if (a.mask) {
                        const uint32_t *mask = a.mask + int64_t(v.t0 + place[r]) * a.mask_words;
                        const int at = j0 >> 5;
                        const uint32_t lo = at < 0 ? ~0u : at < a.mask_words ? mask[at] : 0u, hi = at < -1 ? ~0u : at + 1 < a.mask_words ? mask[at + 1] : 0u;
                        bits &= __funnelshift_r(lo, hi, j0 & 31);
                    } else {
                        bits &= first_bits(place[r] + 1 - j0);
                    }
                }
#pragma unroll
                for (int e = 0; e < OF; ++e) p[r][e] = (bits >> e) & 1u ? p[r][e] : -INFINITY;
                seen[r] = bits;
            }
            // values behind the last key count as 0; are the others finite?
            bool found = false;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t x = w[f][e];
                    if constexpr (OF == 8) {
                        if (k0 + 2 * e + 1 >= end) x &= 0xffffu;
                        if (k0 + 2 * e >= end) x = 0;
                        found |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
                    } else {
                        if (k0 + e >= end) x = 0;
                        found |= (x & 0x7f800000u) == 0x7f800000u;
                    }
                    w[f][e] = x;
                }
            odd = __any(found);
        }

#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = p[r][0];
#pragma unroll
            for (int e = 1; e < OF; ++e) top = fmaxf(top, p[r][e]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float next_m = fmaxf(m[r], top);
            if (__any(next_m > m[r])) {
                const float keep = next_m > m[r] ? exp2_of(m[r] - next_m) : 1.f;   // the first time 2^-inf = 0
                l[r] *= keep;
#pragma unroll
                for (int f = 0; f < NF; ++f) o[r][f] *= keep;
                m[r] = next_m;
            }
            const float from = m[r] == -INFINITY ? 0.f : m[r];   // a row that has seen nothing yet: every weight is 0
#pragma unroll
            for (int e = 0; e < OF; ++e) {
                p[r][e] = exp2_of(p[r][e] - from);
                l[r] += p[r][e];
            }
        }

        u32x4_t pw[RT];   // the weights as operand
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (OF == 8)   // weights in [0, 1] to 8 bits, as the values they multiply
                    pw[r][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{p[r][2 * e], p[r][2 * e + 1]}, bf16x2_t));
                else
                    pw[r][e] = __float_as_uint(p[r][e]);
            }
        if (!odd) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int f = 0; f < NF; ++f) o[r][f] = E::mma(w[f], pw[r], o[r][f]);
        } else {
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                u32x4_t finite, kinds;
                E::part(w[f], finite, kinds);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const f32x4_t counts = E::mma(kinds, E::ones(seen[r]), f32x4_t{0.f, 0.f, 0.f, 0.f});
                    o[r][f] = E::mma(finite, pw[r], o[r][f]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[r][f][e] += limit_of(counts[e]);
                }
                __builtin_amdgcn_sched_barrier(0);   // rare: one piece after another, so that it costs the loop no registers
            }
        }
        if (next < steps) load_v(w, next_page, next_key & (P - 1));
        i = next;
        key = next_key;
        page = next_page;
    }

    // the waves' sums, tile by tile
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float lr = l[r];
        lr += __shfl_xor(lr, 16);
        lr += __shfl_xor(lr, 32);
        __syncthreads();   // the arrays may still be read for the tile before
        if (g == 0) {
            maxima[wave][n] = m[r];
            totals[wave][n] = lr;
        }
        __syncthreads();
        float top = maxima[0][n];
#pragma unroll
        for (int u = 1; u < kWaves; ++u) top = fmaxf(top, maxima[u][n]);
        const float f0 = top == -INFINITY ? 0.f : exp2_of(m[r] - top);
#pragma unroll
        for (int f = 0; f < NF; ++f) *reinterpret_cast<f32x4_t *>(&sums[wave][n][f * 16 + 4 * g]) = o[r][f] * f0;
        __syncthreads();
        for (int j = tid; j < 16 * (DP / 4); j += kThreads) {
            const int rr = j / (DP / 4), d = (j - rr * (DP / 4)) * 4, row = base + r * 16 + rr;
            if (row >= R || (!EVEN && d >= D)) continue;
            float best = maxima[0][rr];
#pragma unroll
            for (int u = 1; u < kWaves; ++u) best = fmaxf(best, maxima[u][rr]);
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
            float total = 0.f;
#pragma unroll
            for (int u = 0; u < kWaves; ++u) {
                sum += *reinterpret_cast<const f32x4_t *>(&sums[u][rr][d]);
                total += best == -INFINITY ? totals[u][rr] : totals[u][rr] * exp2_of(maxima[u][rr] - best);
            }
            const int t = PICKED ? only : row / G;
            const int64_t at = int64_t(v.t0 + t) * H + head * G + (PICKED ? row : row - t * G);
            if (a.n_chunks > 1) {
                const int64_t pa = int64_t(chunk) * a.q.total_q * H + at;
                *reinterpret_cast<f32x4_t *>(a.part_o + pa * D + d) = sum;
                if (d == 0) a.part_ml[pa] = make_float2(best, total);
            } else {
                const float inv = total == 0.f ? 0.f : 1.f / total;
                T *out = static_cast<T *>(a.out) + at * D + d;
#pragma unroll
                for (int e = 0; e < 4; ++e) ElemIO<T>::store(out + e, sum[e] * inv);
                if (d == 0 && a.lse) a.lse[at] = total == 0.f ? -INFINITY : (best + log2f(total)) * kLn2;
            }
        }
    }
}

// Joins the parts of one row: a workgroup per token and head, a wave per part, lanes on channels.
template <typename T, bool PICKED>
__global__ __launch_bounds__(kThreads) void kv_join_kernel(AttentionArgs a, int tile_rows) {
    __shared__ float sums[kWaves][kMaxDim];
    __shared__ float maxima[kWaves], totals[kWaves];
    const int s = blockIdx.z, H = a.q.heads, G = H / a.p.kv_heads, D = a.p.dim;
    const int t = blockIdx.x / H, h = blockIdx.x - t * H, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Span v = span_of(a, s);
    if (t >= v.T) return;
    int parts = a.n_chunks;
    if (!PICKED) {
        const int row = t * G + h % G, last = min(row / tile_rows * tile_rows + tile_rows, v.T * G) - 1;
        parts = max(1, (keys_end(a, v, last, G) + a.chunk - 1) / a.chunk);
    }
    const int64_t at = int64_t(v.t0 + t) * H + h, stride = a.q.total_q * H;
    float m = -INFINITY, l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int c = wave; c < parts; c += kWaves) {
        const float2 ml = a.part_ml[c * stride + at];
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
        if (lane * 4 < D) x = *reinterpret_cast<const f32x4_t *>(a.part_o + (c * stride + at) * D + lane * 4);
        const float top = fmaxf(m, ml.x);
        const float f0 = m == top ? 1.f : exp2_of(m - top), f1 = ml.x == top ? 1.f : exp2_of(ml.x - top);
        o = o * f0 + x * f1;
        l = l * f0 + ml.y * f1;
        m = top;
    }
    if (lane * 4 < D) *reinterpret_cast<f32x4_t *>(&sums[wave][lane * 4]) = o;
    if (lane == 0) {
        maxima[wave] = m;
        totals[wave] = l;
    }
    __syncthreads();
    const int d = threadIdx.x;
    float best = maxima[0], total = 0.f, sum = 0.f;
#pragma unroll
    for (int u = 1; u < kWaves; ++u) best = fmaxf(best, maxima[u]);
#pragma unroll
    for (int u = 0; u < kWaves; ++u) {
        const float f = maxima[u] == best ? 1.f : exp2_of(maxima[u] - best);
        total += totals[u] * f;
        if (d < D) sum += sums[u][d] * f;
    }
    if (d < D) ElemIO<T>::store(static_cast<T *>(a.out) + at * D + d, total == 0.f ? 0.f : sum / total);
    if (d == 0 && a.lse) a.lse[at] = total == 0.f ? -INFINITY : (best + log2f(total)) * kLn2;
}

struct Plan {
    int rt, chunk, n_chunks, row_tiles;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Rows of a workgroup: what the registers hold of queries and sums (RT * 2 * DP / 16 operands of four registers).
int most_tiles(const tbn_kv_pool &p) { return padded_dim(p.dim) == 256 ? 1 : padded_dim(p.dim) == 128 ? 2 : 4; }

Plan plan_of(const tbn_kv_pool &p, int64_t rows, int64_t groups, int64_t units, int64_t unit_step, int64_t unit_most) {
    // units: keys or picks to split, unit_step: the least stretch, a multiple of which a chunk is
    Plan pl;
    pl.rt = 1;
    while (pl.rt * 16 < rows && pl.rt < most_tiles(p)) pl.rt *= 2;
    pl.row_tiles = static_cast<int>(ceil_div(rows, 16 * pl.rt));
    const int64_t blocks = groups * pl.row_tiles;
    const int64_t want = ceil_div(2048, blocks);   // workgroups: several per CU, so that ragged ends even out
    int64_t chunk = ceil_div(ceil_div(units, want), unit_step) * unit_step;
    if (chunk > unit_most) chunk = unit_most;
    pl.chunk = static_cast<int>(chunk);
    pl.n_chunks = static_cast<int>(ceil_div(units, chunk));
    return pl;
}

Plan tree_plan(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q) {
    const int64_t rows = int64_t(q.max_q) * (q.heads / p.kv_heads);
    return plan_of(p, rows, int64_t(ix.n_seqs) * p.kv_heads, q.max_len, 256, int64_t(kListed) * p.page);
}

Plan picked_plan(const tbn_kv_pool &p, const KvQueries &q, int32_t n_select) {
    return plan_of(p, q.heads / p.kv_heads, q.total_q * p.kv_heads, n_select, p.page <= 64 ? 128 / p.page : 1, kListed);
}

size_t workspace_of(const tbn_kv_pool &p, const KvQueries &q, const Plan &pl) {
    return pl.n_chunks > 1 ? static_cast<size_t>(pl.n_chunks) * q.total_q * q.heads * (p.dim + 2) * 4 : 0;
}

template <typename T, int DP, int RT, bool PICKED>
void launch_even(const AttentionArgs &a, dim3 grid, hipStream_t stream) {
    if (a.p.dim == DP) hipLaunchKernelGGL((kv_attention_kernel<T, DP, RT, PICKED, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv_attention_kernel<T, DP, RT, PICKED, false>), grid, dim3(kThreads), 0, stream, a);
}

template <typename T, int DP, bool PICKED>
void launch_tiles(const AttentionArgs &a, int rt, dim3 grid, hipStream_t stream) {
    if constexpr (DP <= 64) {
        if (rt == 4) return launch_even<T, DP, 4, PICKED>(a, grid, stream);
    }
    if constexpr (DP <= 128) {
        if (rt == 2) return launch_even<T, DP, 2, PICKED>(a, grid, stream);
    }
    launch_even<T, DP, 1, PICKED>(a, grid, stream);
}

template <typename T, bool PICKED>
void launch_dims(const AttentionArgs &a, int rt, dim3 grid, dim3 join, hipStream_t stream) {
    switch (padded_dim(a.p.dim)) {
        case 64: launch_tiles<T, 64, PICKED>(a, rt, grid, stream); break;
        case 128: launch_tiles<T, 128, PICKED>(a, rt, grid, stream); break;
        default: launch_tiles<T, 256, PICKED>(a, rt, grid, stream);
    }
    if (a.n_chunks > 1) hipLaunchKernelGGL((kv_join_kernel<T, PICKED>), join, dim3(kThreads), 0, stream, a, 16 * rt);
}

template <bool PICKED>
tbn_status launch(AttentionArgs &a, const Plan &pl, float *ws, const char *what, hipStream_t stream) {
    a.chunk = pl.chunk;
    a.n_chunks = pl.n_chunks;
    a.row_tiles = pl.row_tiles;
    const int64_t parts = int64_t(pl.n_chunks) * a.q.total_q * a.q.heads;
    a.part_o = ws;
    a.part_ml = reinterpret_cast<float2 *>(ws ? ws + parts * a.p.dim : nullptr);
    const int64_t x = int64_t(pl.n_chunks) * pl.row_tiles * (PICKED ? a.q.max_q : 1), jx = int64_t(a.q.max_q) * a.q.heads;
    if (x > 0x7fffffffLL || jx > 0x7fffffffLL) {
        set_error("%s: %lld workgroups per kv head and sequence are beyond one launch", what, (long long)(x > jx ? x : jx));
        return TBN_ERR_UNSUPPORTED;
    }
    const dim3 grid(static_cast<unsigned>(x), a.p.kv_heads, a.ix.n_seqs), join(static_cast<unsigned>(jx), 1, a.ix.n_seqs);
    if (a.p.dt == TBN_F32) launch_dims<float, PICKED>(a, pl.rt, grid, join, stream);
    else launch_dims<uint16_t, PICKED>(a, pl.rt, grid, join, stream);
    return check_launch(what);
}

}  // namespace

size_t tree_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q) { return workspace_of(p, q, tree_plan(p, ix, q)); }

tbn_status launch_tree_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const uint32_t *mask,
                                 int32_t mask_words, float scale, float *ws, hipStream_t stream) {
    AttentionArgs a{p, ix, q, out, lse, mask, mask_words, nullptr, 0, scale * kLog2e};
    return launch<false>(a, tree_plan(p, ix, q), ws, "tbn_tree_attention", stream);
}

size_t block_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &, const KvQueries &q, int32_t n_select) {
    return workspace_of(p, q, picked_plan(p, q, n_select));
}

tbn_status launch_block_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const int32_t *picks,
                                  int32_t n_select, float scale, float *ws, hipStream_t stream) {
    AttentionArgs a{p, ix, q, out, lse, nullptr, 0, picks, n_select, scale * kLog2e};
    return launch<true>(a, picked_plan(p, q, n_select), ws, "tbn_block_attention", stream);
}

}  // namespace tbn
