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
#include <algorithm>
#include <cmath>

#include "tbn_kv_attention.h"

namespace tbn {

namespace {

// RT: row tiles of a workgroup.  DP: channels the registers hold (dim <= DP; EVEN: dim == DP).  TOKENS: blockIdx.y is a token (sequence_of).
template <typename T, int DP, int RT, bool PICKED, bool EVEN, bool TOKENS>
__global__ __launch_bounds__(kAttnThreads, DP == 256 ? 1 : 2) void kv_attention_kernel(AttentionArgs a) {
    using E = Elem<T>;
    constexpr int KS = E::kStep, OF = E::kOf, NF = DP / 16, NQ = NF / E::kTiles;
    __shared__ int2 listed[kListed];   // slot and page
    __shared__ float sums[RT][kAttnWaves][16][DP + 4];
    __shared__ float maxima[kAttnWaves][16], totals[2][kAttnWaves][16];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int s = sequence_of<TOKENS>(a);
    if (TOKENS && s < 0) return;
    const int H = a.q.heads, KV = a.p.kv_heads, G = H / KV, D = EVEN ? DP : a.p.dim, P = a.p.page;
    const int shift = __ffs(P) - 1;
    const Span v = span_of(a, s);
    const Block blk = block_of(a);
    const int head = blk.head, chunk = blk.chunk, only = blk.token, base = blk.row_tile * (16 * RT);
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
        for (int i = tid; i < entries; i += kAttnThreads) {
            const int b = picks[i];
            const bool in = b >= 0 && b < (end + P - 1) >> shift;
            listed[i] = make_int2(in ? b : -1, in ? page_in(table[b], n_pages) : 0);
        }
    } else {
        const int first = chunk * a.chunk;
        if (first >= end && chunk > 0) return;
        entries = (min(end, first + a.chunk) - first + P - 1) >> shift;
        for (int i = tid; i < entries; i += kAttnThreads) {
            const int slot = (first >> shift) + i;
            listed[i] = make_int2(slot, page_in(table[slot], n_pages));
        }
    }

    // this lane's query rows: its token's place and the operand of the first product
    u32x4_t q[RT][NQ];
    int place[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = base + r * 16 + n, in = min(row, R - 1), t = PICKED ? only : in / G;
        place[r] = t;
        const T *src = static_cast<const T *>(a.q.q) + (v.t0 + t) * a.q.q_stride + (head * G + (PICKED ? in : in - t * G)) * D;
        // always loaded, so that the loads do not wait for each other
#pragma unroll
        for (int f = 0; f < NQ; ++f) {
            const int d = f * (4 * OF) + OF * g;
            q[r][f] = *reinterpret_cast<const typename E::u32x4_any *>(src + (EVEN ? d : min(d, D - OF)));
        }
#pragma unroll
        for (int f = 0; f < NQ; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[r][f][e] = row < R && (EVEN || f * (4 * OF) + OF * g < D) ? q[r][f][e] ^ a.flip : 0u;
    }

    f32x4_t o[RT][NF];
    float m[RT], l[RT], z[RT];   // reference, sum of the weights, of the rounded weights (float32: the same, not kept)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY;
        l[r] = z[r] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f) o[r][f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const int64_t page_elems = int64_t(P) * D;
    const T *kp = static_cast<const T *>(a.p.k) + head * page_elems, *vp = static_cast<const T *>(a.p.v) + head * page_elems;
    const int sub_shift = shift - (KS == 32 ? 5 : 4);
    const int steps = entries << sub_shift;
    // piece f of K: bfloat16 tile f % 2, channels 32 (f / 2) + 8 g; row n of tile 0 / 1 is key 8 (n / 4) + n % 4 (+ 4)
    const int k_key = OF == 8 ? 8 * (n >> 2) + (n & 3) : n;
    // one lane offset for all pieces of K, one for all of V; what differs between pieces is the same for all lanes
    const uint32_t k_lane = (k_key * D + OF * g) * sizeof(T), v_lane = (n * P + OF * g) * sizeof(T);
    auto load_k = [&](u32x4_t (&k)[NF], int page, int off) {
        const T *src = kp + int64_t(page) * (page_elems * KV) + off * D;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int d = OF == 8 ? (f / 2) * 32 : f * 16;
            const char *at = reinterpret_cast<const char *>(src + d + (OF == 8 ? (f & 1) * 4 * D : 0));
            u32x4_t w = {0, 0, 0, 0};
            if (EVEN || d + OF * g < D) w = *reinterpret_cast<const u32x4_t *>(at + k_lane);
            k[f] = w;
        }
    };
    auto load_v = [&](u32x4_t (&w)[NF], int page, int off) {
        const T *src = vp + int64_t(page) * (page_elems * KV) + off;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const char *at = reinterpret_cast<const char *>(src + f * 16 * P);
            u32x4_t x = {0, 0, 0, 0};
            if (EVEN || f * 16 + n < D) x = *reinterpret_cast<const u32x4_t *>(at + v_lane);
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
            i += kAttnWaves;
        }
        return i;
    };

    bool any_odd = false;   // of this wave
    auto clear_limits = [&] {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll 1
            for (int f = 0; f < NF; ++f) *reinterpret_cast<f32x4_t *>(&sums[r][wave][n][f * 16 + 4 * g]) = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
        const int next = next_step(i + kAttnWaves, next_key, next_page);
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
                // four short chains round less than a long one: relative error of the result 4e-7 instead of 1.1e-6 (256 channels, 1814 keys), in the same time
                f32x4_t s2 = {0.f, 0.f, 0.f, 0.f}, s3 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < NF; f += 4) {
                    s0 = E::mma(k[f], q[r][f], s0);
                    s1 = E::mma(k[f + 1], q[r][f + 1], s1);
                    s2 = E::mma(k[f + 2], q[r][f + 2], s2);
                    s3 = E::mma(k[f + 3], q[r][f + 3], s3);
                }
                s0 = (s0 + s1) + (s2 + s3);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[r][e] = s0[e];
                if constexpr (OF == 8) p[r][4 + e] = s1[e];
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
                const uint32_t bits = seen_bits<PICKED>(a, v, k0, end, place[r]);
#pragma unroll
                for (int e = 0; e < OF; ++e) p[r][e] = (bits >> e) & 1u ? p[r][e] : -INFINITY;
                seen[r] = bits;
            }
            // values behind the last key count as 0; are the others finite?
            bool found = false;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                w[f] = E::first_of(w[f], end - k0);
                found |= E::not_finite(w[f]);
            }
            odd = __any(found);
        }

#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = p[r][0];
#pragma unroll
            for (int e = 1; e < OF; ++e) top = fmaxf(top, p[r][e]);
            top = max_over_32(max_over_16(top)) * a.c;
            if (__any(top > m[r] + kSlack)) {
                const float next_m = fmaxf(m[r], top), keep = next_m > m[r] ? exp2_of(m[r] - next_m) : 1.f;   // the first time 2^-inf = 0
                l[r] *= keep;
                z[r] *= keep;
#pragma unroll
                for (int f = 0; f < NF; ++f) o[r][f] *= keep;
                m[r] = next_m;
            }
            const float from = reference_of(m[r]);
#pragma unroll
            for (int e = 0; e < OF; ++e) {
                p[r][e] = exp2_of(fmaf(p[r][e], a.c, -from));
                l[r] += p[r][e];
            }
        }

        u32x4_t pw[RT];   // the weights as operand
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (OF == 8) {
                    pw[r][e] = two_bf16(p[r][2 * e], p[r][2 * e + 1]);
                    z[r] = add_two_bf16(pw[r][e], z[r]);
                } else {
                    pw[r][e] = __float_as_uint(p[r][e]);
                }
            }
        if (odd) {   // rare: what such values add to the rows that see them goes to LDS until the end, and 0 in their place
            if (!any_odd) clear_limits();
            any_odd = true;
            const T *src = vp + int64_t(page) * (page_elems * KV) + (key & (P - 1)) + OF * g;
#pragma unroll 1
            for (int f = 0; f < NF; ++f) {   // loaded again: a loop that is not unrolled costs the others no registers
                const int d = f * 16 + n;
                u32x4_t x = {0, 0, 0, 0}, finite, kinds;
                if (EVEN || d < D) x = E::first_of(*reinterpret_cast<const u32x4_t *>(src + d * P), end - key - OF * g);
                E::part(x, finite, kinds);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const f32x4_t counts = E::mma(kinds, E::ones(seen[r]), f32x4_t{0.f, 0.f, 0.f, 0.f});
                    float *limit = &sums[r][wave][n][f * 16 + 4 * g];
#pragma unroll
                    for (int e = 0; e < 4; ++e) limit[e] += limit_of(counts[e]);
                }
            }
#pragma unroll
            for (int f = 0; f < NF; ++f) w[f] = E::finite_of(w[f]);
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int f = 0; f < NF; ++f) o[r][f] = E::mma(w[f], pw[r], o[r][f]);
        if (next < steps) load_v(w, next_page, next_key & (P - 1));
        i = next;
        key = next_key;
        page = next_page;
    }

    // the waves' sums, tile by tile
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float lr = l[r], zr = OF == 8 ? z[r] : l[r];
        lr += __shfl_xor(lr, 16);
        lr += __shfl_xor(lr, 32);
        zr += __shfl_xor(zr, 16);
        zr += __shfl_xor(zr, 32);
        __syncthreads();   // the arrays may still be read for the tile before
        if (g == 0) {
            maxima[wave][n] = m[r];
            totals[0][wave][n] = lr;
            totals[1][wave][n] = zr;
        }
        __syncthreads();
        float top = maxima[0][n];
#pragma unroll
        for (int u = 1; u < kAttnWaves; ++u) top = fmaxf(top, maxima[u][n]);
        const float f0 = m[r] == top ? 1.f : exp2_of(m[r] - top);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            f32x4_t *at = reinterpret_cast<f32x4_t *>(&sums[r][wave][n][f * 16 + 4 * g]), sum = o[r][f] * f0;
            if (any_odd) sum += *at;
            *at = sum;
        }
        __syncthreads();
        for (int j = tid; j < 16 * (DP / 4); j += kAttnThreads) {
            const int rr = j / (DP / 4), d = (j - rr * (DP / 4)) * 4, row = base + r * 16 + rr;
            if (row >= R || (!EVEN && d >= D)) continue;
            float best = maxima[0][rr];
#pragma unroll
            for (int u = 1; u < kAttnWaves; ++u) best = fmaxf(best, maxima[u][rr]);
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
            float lsum = 0.f, zsum = 0.f;
#pragma unroll
            for (int u = 0; u < kAttnWaves; ++u) {
                const float f = maxima[u][rr] == best ? 1.f : exp2_of(maxima[u][rr] - best);
                lsum += totals[0][u][rr] * f;
                zsum += totals[1][u][rr] * f;
                sum += *reinterpret_cast<const f32x4_t *>(&sums[r][u][rr][d]);
            }
            const int t = PICKED ? only : row / G;
            const int64_t at = int64_t(v.t0 + t) * H + head * G + (PICKED ? row : row - t * G);
            store_sums<T>(a, chunk, at, d, sum, best, lsum, zsum);
        }
    }
}

// Joins the parts of one row.  D / 4 lanes (rounded up to a power of two) take a part at a time.  WIDE: a workgroup per row, else a wave.
template <typename T, bool PICKED, bool WIDE, bool TOKENS>
__global__ __launch_bounds__(kAttnThreads) void kv_join_kernel(AttentionArgs a, int tile_rows) {
    constexpr int kTeam = WIDE ? kAttnThreads : kWave;
    __shared__ f32x4_t sums[WIDE ? kAttnThreads : 1];
    __shared__ float maxima[kAttnWaves];
    __shared__ float2 totals[WIDE ? kAttnThreads / 16 : 1];
    const int s = sequence_of<TOKENS>(a);
    if (TOKENS && s < 0) return;
    const int H = a.q.heads, G = H / a.p.kv_heads, D = a.p.dim, tid = threadIdx.x % kTeam;
    const int row = WIDE ? blockIdx.x : __builtin_amdgcn_readfirstlane(blockIdx.x * kAttnWaves + threadIdx.x / kWave);
    const int t = row / H, h = row - t * H;
    const Span v = span_of(a, s);
    if (t >= v.T) return;
    int parts = a.n_chunks;
    if (!PICKED) {
        const int r = t * G + h % G, last = min(r / tile_rows * tile_rows + tile_rows, v.T * G) - 1;
        parts = max(1, (keys_end(a, v, last, G) + a.chunk - 1) / a.chunk);
    }
    const int64_t at = int64_t(v.t0 + t) * H + h, stride = a.q.total_q * H;
    const int shift = D <= 64 ? 4 : D <= 128 ? 5 : 6, group = tid >> shift, groups = kTeam >> shift, d = (tid & ((1 << shift) - 1)) * 4;
    // the first parts' sums are on their way while the maximum is found (13 tokens on 7 sequences of 1009 keys, float32: 12.5 us with both
    // kernels, 13.3 without; bfloat16 cases level)
    constexpr int kAhead = 4;
    float4 first_ml[kAhead];
    f32x4_t first_o[kAhead];
    const float *from = a.part_o + at * D + min(d, D - 4);   // lanes beyond the head's channels: any, their sums are dropped
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int c = min(group + j * groups, parts - 1);
        first_ml[j] = a.part_ml[c * stride + at];
        first_o[j] = *reinterpret_cast<const f32x4_t *>(from + c * stride * D);
    }
    float best = -INFINITY;
    for (int c = tid; c < parts; c += kTeam) best = fmaxf(best, a.part_ml[c * stride + at].x);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) best = fmaxf(best, __shfl_xor(best, d));
    if constexpr (WIDE) {
        if ((tid & 63) == 0) maxima[tid >> 6] = best;
        __syncthreads();
        best = fmaxf(fmaxf(maxima[0], maxima[1]), fmaxf(maxima[2], maxima[3]));
    }
    float l = 0.f, z = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float4 &ml, const f32x4_t &x) {
        const float f = ml.x == best ? 1.f : exp2_of(ml.x - best);   // no part has seen a key: every sum is 0
        o += x * f;
        l += ml.y * f;
        z += ml.z * f;
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (group + j * groups < parts) add(first_ml[j], first_o[j]);
#pragma unroll 4
    for (int c = group + kAhead * groups; c < parts; c += groups) add(a.part_ml[c * stride + at], *reinterpret_cast<const f32x4_t *>(from + c * stride * D));
    if constexpr (WIDE) {
        sums[tid] = o;
        if (d == 0) totals[group] = make_float2(l, z);
        __syncthreads();
        if (group > 0) return;
        for (int g = 1; g < groups; ++g) {
            o += sums[(g << shift) + tid];
            l += totals[g].x;
            z += totals[g].y;
        }
    } else {
        for (int x = 1 << shift; x < kWave; x <<= 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x);
            l += __shfl_xor(l, x);
            z += __shfl_xor(z, x);
        }
        if (group > 0) return;
    }
    if (d < D) {
        const float inv = z == 0.f ? 0.f : 1.f / z;
        T *out = static_cast<T *>(a.out) + at * D + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) ElemIO<T>::store(out + e, o[e] * inv);
    }
    if (tid == 0 && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (best + log2f(l)) * kLn2;
}

template <typename T, bool PICKED, bool TOKENS>
void launch_join(const AttentionArgs &a, int tile_rows, unsigned groups, hipStream_t stream) {
    const int64_t rows = int64_t(a.q.max_q) * a.q.heads;   // checked by the caller
    // many parts of a row: a workgroup each; few: a wave each (13000 rows of at most 4 parts: 14 us with a workgroup each)
    if (a.n_chunks > 16) hipLaunchKernelGGL((kv_join_kernel<T, PICKED, true, TOKENS>), dim3(static_cast<unsigned>(rows), groups), dim3(kAttnThreads), 0, stream, a, tile_rows);
    else hipLaunchKernelGGL((kv_join_kernel<T, PICKED, false, TOKENS>), dim3(static_cast<unsigned>((rows + kAttnWaves - 1) / kAttnWaves), groups), dim3(kAttnThreads), 0, stream, a, tile_rows);
}

struct Plan {
    int rows, chunk, n_chunks, row_tiles;   // rows of a workgroup: 16 (float32 up to 64) in this file's kernel, 64 or 128 in the one for many rows
    bool staged;                            // the latter
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Rows of a workgroup of this file's kernel: what the registers hold of queries and sums.  (bfloat16: more rows go to the other kernel.)
int most_rows(const tbn_kv_pool &p) { return p.dt == TBN_BF16 || padded_dim(p.dim) == 256 ? 16 : padded_dim(p.dim) == 128 ? 32 : 64; }

Plan plan_of(const tbn_kv_pool &p, int64_t rows, int64_t groups, int64_t units, int64_t unit_step, int64_t unit_most, bool picked) {
    // units: keys or picks to split, unit_step: the least stretch, a multiple of which a chunk is
    Plan pl;
    const int64_t places = padded_dim(p.dim) == 256 ? 256 : 512;   // for workgroups at a time: the least of both kernels
    // groups: sequences of the call (of picked blocks: queries) x kv heads
    // fill: keys that give each place for a workgroup one stretch.  Short sequences that fill the CUs are not split.
    const double fill = static_cast<double>(units) * groups / places;
    const bool whole = units <= 1024 && groups >= 256;
    // one round of the staged kernel: as many stretches as fit, where they take 7/8 of the places; otherwise a few more than fit
    const int64_t fit = places / groups;
    const bool round = fit * groups * 8 >= places * 7;
    // Up to 16 rows and 128 channels the staged kernel's waves read each byte of the cache for one another and its loads run further ahead: it is
    // the faster one as soon as each place has more than 256 keys of its own and one round takes the work (16 sequences of 16000 keys,
    // 4 - 7 rows: 130 us, 143 - 150 in the other; 8 of 3000, 22 to 26; 100 of 1500 with 16 rows, 95 to 114).  Below, and where a round ends
    // half full, the other one's short stretches win (4 of 2000: 14.1 us to 15.0; 34 of 3698: 79 to 92; 200 of 300: 45 to 59).  With 64
    // and 256 channels they measure alike.
    const bool few = rows <= 16 && padded_dim(p.dim) == 128 && p.dim > 96 && fill > 256 && !whole && (groups >= places || round);
    pl.staged = !picked && p.dt == TBN_BF16 && (rows > 16 || few);
    if (pl.staged) {
        pl.rows = rows <= 64 ? 64 : 128;
    } else {
        pl.rows = 16;
        while (pl.rows < rows && pl.rows < most_rows(p)) pl.rows *= 2;
    }
    pl.row_tiles = static_cast<int>(ceil_div(rows, pl.rows));
    const int64_t blocks = groups * pl.row_tiles;
    // Stretches of keys.  The staged kernel takes one round of the places (64 drafted tokens on 131000 keys: 188 us, in four rounds 227).  Two where
    // whole sequences of few rows would fill the round and are long: their lengths are ragged, and halves of them even that out (64 sequences of
    // 4096 - 16384 keys: 456 us, 490 in one round, 462 in the other kernel; up to 8192: 236 - 242, 250 in one; 4100: 133 - 139 to 135 - 142; 3200 level; 100 of
    // 2000: 119 - 123 to 110 - 113).  Fewer sequences are cut into more stretches anyway (16 of 60000: 410 - 425 us in one round, 431 - 454 in two; 32 of
    // 16384 level).  Here many short stretches even them out, against the cost of starting, ending and joining each.
    const int64_t parts = (few && round ? fit : ceil_div(places, blocks)) * (few && groups >= places && units > 4096 ? 2 : 1);
    int64_t chunk = ceil_div(units, pl.staged ? parts : ceil_div(8192, blocks));
    if (!picked && !pl.staged) {
        // Beyond 256 keys several stretches a place: with a cost of c keys each and about half a stretch idle at the end, the best length grows
        // as sqrt(2 c fill); c of 32 was measured (34 sequences of up to 3698 keys, float32: 72 us with 256 keys, 97 with 1024; 16 of 16000,
        // 16 rows: 155 us with 512 - 1024, 168 with 256).  Below, the nearest multiple of a step of each wave (9 sequences of 15000 keys: 18.9 us
        // with 256 keys, 21.7 with 384, 22.5 with 128).
        const double want = fill * pl.row_tiles <= 256 ? fill * pl.row_tiles : std::fmax(256, std::fmin(1024, 8 * std::sqrt(fill * pl.row_tiles)));
        const int64_t least = static_cast<int64_t>(want / unit_step + 0.5) * unit_step;
        if (chunk < least) chunk = least;
        // not split, the join would take longer (40 sequences of 600 keys, 8 kv heads: 20 us, 24 in parts)
        if (units <= 1024 && blocks >= 256) chunk = units;
    }
    // Nor up to 80 KB of keys: the join's launch takes longer than the steps it saves (one sequence, 8 kv heads of 128 channels, bfloat16: 200
    // keys 8.0 us, 10.2 in parts; 300 keys 9.3 to 10.2; 513 keys 12.4 to 10.4).
    if (!pl.staged && units * (picked ? p.page : 1) * padded_dim(p.dim) * (p.dt == TBN_F32 ? 4 : 2) <= 80 * 1024) chunk = units;
    chunk = ceil_div(chunk, unit_step) * unit_step;
    if (chunk > unit_most) chunk = unit_most;
    pl.chunk = static_cast<int>(chunk);
    pl.n_chunks = static_cast<int>(ceil_div(units, chunk));
    return pl;
}

// Whether a launch has a row of workgroups per token of the call instead of per place of the index (sequence_of): where no token is without work, or
// places are many more.
bool by_token(const tbn_kv_index &ix, const KvQueries &q) { return q.total_q < ix.n_seqs && (q.max_q == 1 || 16 * q.total_q <= ix.n_seqs); }

// Workgroups of a launch whose rows may mostly be idle, at most: 0.2 - 0.6 ns each where they end at once, small against the work.
double most_blocks(const KvQueries &q) { return std::min(150000., 16384. + 8. * q.max_len); }

// An index has room for more sequences than are there, so keys are split by the sequences of the call: max_q tokens each would be the fewest; drafts are
// ragged, half of max_q and more in the mean, so twice that (16 trees of up to 26 tokens: 49 us, 58 with the fewest).  One token on 131000 keys in one of 64
// places: 101 us, 1065 split by places; a tree of 26: 124 and 1383.  But every place (or token, whose idle workgroups take five times as long) has its row
// of workgroups: beyond most_blocks they are split as if for twice as many sequences, and so on up to one for each row.
Plan tree_plan(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q) {
    const int64_t rows = int64_t(q.max_q) * (q.heads / p.kv_heads);
    const bool token = by_token(ix, q);
    const int64_t most = token ? q.total_q : ix.n_seqs;
    const double weight = most * (token && q.max_q > 1 ? 5. : 1.), join = double(q.max_q) * q.heads;
    int64_t sequences = std::min<int64_t>({ix.n_seqs, q.total_q, 2 * ceil_div(q.total_q, q.max_q)});
    for (;; sequences = std::min(most, 2 * sequences)) {
        const Plan pl = plan_of(p, rows, sequences * p.kv_heads, q.max_len, 128, int64_t(kListed) * p.page, false);
        const double blocks = double(pl.n_chunks) * pl.row_tiles * p.kv_heads + (pl.n_chunks > 16 ? join : pl.n_chunks > 1 ? join / 4 : 0.);
        if (sequences >= most || blocks * weight <= most_blocks(q)) return pl;
    }
}

Plan picked_plan(const tbn_kv_pool &p, const KvQueries &q, int32_t n_select) {
    return plan_of(p, q.heads / p.kv_heads, q.total_q * p.kv_heads, n_select, p.page <= 64 ? 128 / p.page : 1, kListed, true);
}

size_t workspace_of(const tbn_kv_pool &p, const KvQueries &q, const Plan &pl) {
    return pl.n_chunks > 1 ? static_cast<size_t>(pl.n_chunks) * q.total_q * q.heads * (p.dim + 4) * 4 : 0;
}

template <typename T, int DP, int RT, bool PICKED, bool TOKENS>
void launch_even(const AttentionArgs &a, dim3 grid, hipStream_t stream) {
    if (a.p.dim == DP) hipLaunchKernelGGL((kv_attention_kernel<T, DP, RT, PICKED, true, TOKENS>), grid, dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv_attention_kernel<T, DP, RT, PICKED, false, TOKENS>), grid, dim3(kAttnThreads), 0, stream, a);
}

template <typename T, int DP, bool PICKED, bool TOKENS>
void launch_rows(const AttentionArgs &a, int rows, dim3 grid, hipStream_t stream) {
    if constexpr (sizeof(T) == 4 && DP <= 64) {
        if (rows == 64) return launch_even<T, DP, 4, PICKED, TOKENS>(a, grid, stream);
    }
    if constexpr (sizeof(T) == 4 && DP <= 128) {
        if (rows == 32) return launch_even<T, DP, 2, PICKED, TOKENS>(a, grid, stream);
    }
    launch_even<T, DP, 1, PICKED, TOKENS>(a, grid, stream);
}

// Both kernels; pl.staged: the first one is another file's.
template <typename T, bool PICKED, bool TOKENS>
void launch_both(const AttentionArgs &a, const Plan &pl, dim3 grid, hipStream_t stream) {
    if (pl.staged) launch_kv_rows(a, pl.rows / 32, TOKENS, grid, stream);
    else if (padded_dim(a.p.dim) == 64) launch_rows<T, 64, PICKED, TOKENS>(a, pl.rows, grid, stream);
    else if (padded_dim(a.p.dim) == 128) launch_rows<T, 128, PICKED, TOKENS>(a, pl.rows, grid, stream);
    else launch_rows<T, 256, PICKED, TOKENS>(a, pl.rows, grid, stream);
    if (a.n_chunks > 1) launch_join<T, PICKED, TOKENS>(a, pl.rows, grid.y, stream);
}

template <bool PICKED, bool TOKENS>
void launch_type(const AttentionArgs &a, const Plan &pl, dim3 grid, hipStream_t stream) {
    if (a.p.dt == TBN_F32) launch_both<float, PICKED, TOKENS>(a, pl, grid, stream);
    else launch_both<uint16_t, PICKED, TOKENS>(a, pl, grid, stream);
}

float factor_of(float scale) {
    const float c = fabsf(scale) * kLog2e;
    return c < 1e-37f ? 1e-37f : c;
}
uint32_t flip_of(const tbn_kv_pool &p, float scale) { return !(scale < 0.f) ? 0u : p.dt == TBN_F32 ? 0x80000000u : 0x80008000u; }

constexpr int64_t kMostBlocks = 0x7fffffff;   // workgroups of a sequence

tbn_status too_many(const char *what, int64_t blocks) {
    set_error("%s: %lld workgroups per sequence are beyond one launch", what, (long long)blocks);
    return TBN_ERR_UNSUPPORTED;
}

template <bool PICKED>
tbn_status launch(AttentionArgs &a, const Plan &pl, float *ws, const char *what, hipStream_t stream) {
    a.chunk = pl.chunk;
    a.n_chunks = pl.n_chunks;
    a.row_tiles = pl.row_tiles;
    const int64_t parts = int64_t(pl.n_chunks) * a.q.total_q * a.q.heads;
    a.part_o = ws;
    a.part_ml = reinterpret_cast<float4 *>(ws ? ws + parts * a.p.dim : nullptr);
    const int64_t x = int64_t(pl.n_chunks) * pl.row_tiles * a.p.kv_heads * (PICKED ? a.q.max_q : 1), jx = int64_t(a.q.max_q) * a.q.heads;
    if (x > kMostBlocks || jx > kMostBlocks) return too_many(what, x > jx ? x : jx);
    if constexpr (!PICKED) {
        if (by_token(a.ix, a.q)) {
            launch_type<false, true>(a, pl, dim3(static_cast<unsigned>(x), static_cast<unsigned>(a.q.total_q)), stream);
            return check_launch(what);
        }
    }
    launch_type<PICKED, false>(a, pl, dim3(static_cast<unsigned>(x), a.ix.n_seqs), stream);
    return check_launch(what);
}

}  // namespace

size_t tree_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q) { return workspace_of(p, q, tree_plan(p, ix, q)); }

tbn_status launch_tree_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const uint32_t *mask,
                                 int32_t mask_words, float scale, float *ws, hipStream_t stream) {
    AttentionArgs a{p, ix, q, out, lse, mask, mask_words, nullptr, 0, factor_of(scale), flip_of(p, scale)};
    return launch<false>(a, tree_plan(p, ix, q), ws, "tbn_tree_attention", stream);
}

size_t block_attention_workspace(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_select) {
    return picked_queries(p, ix, q, n_select) ? 0 : workspace_of(p, q, picked_plan(p, q, n_select));
}

tbn_status launch_block_attention(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, void *out, float *lse, const int32_t *picks,
                                  int32_t n_select, float scale, float *ws, hipStream_t stream) {
    AttentionArgs a{p, ix, q, out, lse, nullptr, 0, picks, n_select, factor_of(scale), flip_of(p, scale)};
    const char *what = "tbn_block_attention";
    if (const int queries = picked_queries(p, ix, q, n_select)) {
        a.n_chunks = 1;
        a.row_tiles = static_cast<int>(ceil_div(q.max_q, queries));
        const int64_t x = int64_t(a.row_tiles) * p.kv_heads;
        if (x > kMostBlocks) return too_many(what, x);
        launch_kv_picked(a, queries, dim3(static_cast<unsigned>(x), ix.n_seqs), stream);
        return check_launch(what);
    }
    return launch<true>(a, picked_plan(p, q, n_select), ws, what, stream);
}

}  // namespace tbn
