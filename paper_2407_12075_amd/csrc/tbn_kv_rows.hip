// Attention of many rows (drafted trees, prompt chunks; bfloat16) over the paged cache.  Mathematics, masks and parts as in
// tbn_kv_attention.hip; here the rows are so many that the matrix cores and not the cache's bytes are the bound, so the keys
// are staged in LDS once for all waves of a workgroup.  Few rows on enough keys to give every CU a long stretch come here too: loads that need no
// registers run further ahead (16 sequences of 16000 keys, 8 kv heads of 128 channels, one token: 129 us, 5.5 TB/s; 143 us in the other kernel).
//
// A workgroup takes 64 or 128 rows.  Four waves with 32 rows each (two with 64 rows: the waves of a pair take alternate halves of
// the keys and are merged at the end) go through the keys 64 at a time.  Both products are v_mfma_f32_32x32x16_bf16 with the query
// rows as columns:
//
//   S^T = K Q^T   (lane l: row l % 32; of 32 keys the 16 with (key / 8) % 2 = l / 32)
//   O^T += V^T P^T
//
// As there, rows of K are dealt to the instruction's rows so that a lane's eight logits in a row belong to eight neighbouring keys:
// the weights are the second product's operand where they arise, and a row's maximum is one exchange between two lanes.
//
// K and V^T tiles go from memory to LDS without passing through registers, one step ahead; a tile's 16-byte pieces are permuted
// within its rows (piece index xor row) by the addresses they are loaded from, so that the eight lanes that read LDS together hit
// eight different places.
#include "tbn_kv_attention.h"

namespace tbn {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};   // pieces beyond the head's channels

__device__ __forceinline__ f32x16_t mma(u32x4_t a, u32x4_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Every wave has done its accesses to LDS.  Loads into it may still be on their way, which __syncthreads would wait for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// key of row r of a tile of 32: the instruction's output register 4 i + j of a lane of half h is row 8 i + 4 h + j
__device__ __forceinline__ int key_of_row(int r) { return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3); }

// DP: channels (dim <= DP; EVEN: equal).  RW: groups of 32 rows, 4 / RW waves each.  TOKENS: blockIdx.y is a token (sequence_of).
template <int DP, int RW, Kind KIND, bool EVEN, bool TOKENS>
__global__ __launch_bounds__(kAttnThreads, DP == 256 ? 1 : 2) void kv_rows_kernel(AttentionArgs a) {
    constexpr bool WINDOW = KIND == kWindow;
    constexpr int KW = kAttnWaves / RW, KEYS = DP == 256 && KW == 1 ? 32 : 64, TILES = KEYS / 32 / KW;
    constexpr int PITCH = DP == 96 ? 128 : DP;                     // channels of a row of K in LDS
    constexpr bool FULL = EVEN && PITCH == DP;                     // every piece of such a row is the head's
    constexpr int KP = PITCH / 8, VP = KEYS / 8;                   // 16-byte pieces of a row of K, of V^T
    constexpr int NK = KEYS * KP / kAttnThreads, NV = DP * VP / kAttnThreads;
    constexpr int NQ = DP / 16, ND = DP / 32;
    // two buffers of each, as arrays of their own: the compiler then knows that reads of one do not wait for loads into the other
    __shared__ __attribute__((aligned(16))) uint16_t k0[KEYS * PITCH], k1[KEYS * PITCH], v0[DP * KEYS], v1[DP * KEYS];
    __shared__ int listed[kListed];
    __shared__ float4 halves[RW][32];
    __shared__ int odd_seen;   // with a window: whether a step that not every row sees all of has a value that is not finite

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int s = sequence_of<TOKENS>(a);
    if (TOKENS && s < 0) return;
    const int H = a.q.heads, KV = a.p.kv_heads, G = H / KV, D = EVEN ? DP : a.p.dim, P = a.p.page;
    const int shift = __ffs(P) - 1, group = wave % RW, half = wave / RW;
    const Span v = span_of(a, s);
    const Block blk = block_of(a);
    const int R = v.T * G, base = blk.row_tile * (32 * RW);
    if (base >= R) return;
    // a window's keys are counted along the pages that are gone through
    const int last = min(base + 32 * RW, R) - 1;
    Within in_reach = {};
    if constexpr (WINDOW) in_reach = within_of(a, v, base, last, G, shift);
    const int end = WINDOW ? in_reach.end : keys_end(a, v, last, G);
    const int first = blk.chunk * a.chunk;
    if (first >= end && blk.chunk > 0) return;
    const int stop = min(end, first + a.chunk), entries = (stop - first + P - 1) >> shift;
    const int32_t *table = a.ix.table + int64_t(s) * a.ix.max_pages + (WINDOW ? 0 : first >> shift);
    for (int i = tid; i < entries; i += kAttnThreads)
        listed[i] = page_in(table[WINDOW ? in_reach.key(first + (i << shift)) >> shift : i], static_cast<int>(a.p.n_pages));

    const int row = base + group * 32 + n, in = min(row, R - 1), place = in / G;
    const int low = WINDOW ? window_of(a, v, place) : 0;
    const int64_t at = int64_t(v.t0 + place) * H + blk.head * G + (in - place * G);   // of the outputs, where row < R
    u32x4_t q[NQ];
    {
        const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (v.t0 + place) * a.q.q_stride + (blk.head * G + in - place * G) * D;
        // always loaded, so that the loads do not wait for each other
#pragma unroll
        for (int f = 0; f < NQ; ++f) q[f] = *reinterpret_cast<const Elem<uint16_t>::u32x4_any *>(src + (EVEN ? f * 16 + 8 * h : min(f * 16 + 8 * h, D - 8)));
#pragma unroll
        for (int f = 0; f < NQ; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[f][e] = row < R && (EVEN || f * 16 + 8 * h < D) ? q[f][e] ^ a.flip : 0u;
    }

    // where this lane's pieces come from: offsets within a page in bytes, relative to the step's first key
    const int64_t page_elems = int64_t(P) * D;
    const uint16_t *kp = static_cast<const uint16_t *>(a.p.k) + blk.head * page_elems, *vp = static_cast<const uint16_t *>(a.p.v) + blk.head * page_elems;
    uint32_t k_from[NK], v_from[NV];
    bool k_there[NK];
#pragma unroll
    for (int j = 0; j < NK; ++j) {
        const int L = (j * kAttnWaves + wave) * kWave + lane, r = L / KP, c = (L % KP) ^ (r & 7);
        k_from[j] = (((r & ~31) + key_of_row(r & 31)) * D + c * 8) * 2;
        k_there[j] = FULL || c * 8 < D;
    }
    auto v_swap = [](int d) { return KEYS == 64 ? d & 7 : (d >> 1) & 3; };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int L = (j * kAttnWaves + wave) * kWave + lane, d = L / VP, c = (L % VP) ^ v_swap(d);
        v_from[j] = (min(d, D - 1) * P + c * 8) * 2;   // channels beyond the head's: any, their sums are dropped
    }
    const bool late = ((lane % VP) ^ v_swap(lane / VP)) * 8 >= 32;   // this lane's pieces of V lie in the second 32 keys of a step (the same for all j)
    typedef __attribute__((address_space(1))) const void *global_ptr;
    typedef __attribute__((address_space(3))) void *lds_ptr;
    auto request = [&](int i, uint16_t *kt, uint16_t *vt) {
        const int off = i * KEYS, e = min(off >> shift, entries - 1), in = off & (P - 1);
        const int page = __builtin_amdgcn_readfirstlane(listed[e]);
        int later = page;
        if (KEYS > 32 && P == 32) later = __builtin_amdgcn_readfirstlane(listed[min(e + 1, entries - 1)]);
        const char *ka = reinterpret_cast<const char *>(kp + int64_t(page) * (page_elems * KV) + in * D), *va = reinterpret_cast<const char *>(vp + int64_t(page) * (page_elems * KV) + in);
        const char *kb = ka, *vb = va;
        if (KEYS > 32 && P == 32) {   // the second 32 keys of a step are another page's first
            kb = reinterpret_cast<const char *>(kp + int64_t(later) * (page_elems * KV) - 32 * D);
            vb = reinterpret_cast<const char *>(vp + int64_t(later) * (page_elems * KV) - 32);
        }
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const char *from = ((j * kAttnThreads) / KP >= 32 ? kb : ka) + k_from[j];
            if (!FULL) from = k_there[j] ? from : reinterpret_cast<const char *>(kZeros);
            __builtin_amdgcn_global_load_lds((global_ptr)from, (lds_ptr)(kt + (j * kAttnWaves + wave) * (kWave * 8)), 16, 0, 0);
        }
        const char *vl = late ? vb : va;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            __builtin_amdgcn_global_load_lds((global_ptr)(vl + v_from[j]), (lds_ptr)(vt + (j * kAttnWaves + wave) * (kWave * 8)), 16, 0, 0);
    };

    f32x16_t o[ND];
#pragma unroll
    for (int f = 0; f < ND; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[f][e] = 0.f;
    float m = -INFINITY, l = 0.f, z = 0.f;
    const int all_see = a.mask ? v.prefix : v.prefix + base / G + 1;   // keys from here on are not seen by every row
    const int all_from = WINDOW ? last_window(a, v, last, G) : 0;                  // keys before this one, the first ones aside, neither
    // which of eight keys, counted as the steps are, this lane's row sees
    auto seen = [&](int x) {
        const int k = WINDOW ? in_reach.key(x) : x;
        return seen_within<KIND>(a, v, k, stop + (k - x), place, low);
    };

    auto compute = [&](int i, const uint16_t *kt, uint16_t *vt) {
        f32x16_t p[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) p[t][e] = 0.f;
#pragma unroll
        for (int f = 0; f < NQ; ++f)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                p[t] = mma(*reinterpret_cast<const u32x4_t *>(kt + ((KW > 1 ? half : t) * 32 + n) * PITCH + ((2 * f + h) ^ (n & 7)) * 8), q[f], p[t]);
        const int key = first + i * KEYS;
        bool edge = key + KEYS > stop;   // the same for all lanes
        if constexpr (WINDOW) {
#pragma unroll
            for (int t = 0; t < KEYS; t += 32) {
                const int k = in_reach.key(key + t);
                edge |= k + 32 > all_see || (k < all_from && k + 32 > a.window.sink);
            }
        } else {
            edge |= key + KEYS > all_see;
        }
        if (edge) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t bits = seen(key + (KW > 1 ? half : t) * 32 + 16 * u + 8 * h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[t][8 * u + e] = (bits >> e) & 1u ? p[t][8 * u + e] : -INFINITY;
                }
        }
        float top = p[0][0];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, p[t][e]);
        top = max_over_32(top) * a.c;
        if (__any(top > m + kSlack)) {
            const float next_m = fmaxf(m, top), keep = next_m > m ? exp2_of(m - next_m) : 1.f;
            l *= keep;
            z *= keep;
#pragma unroll
            for (int f = 0; f < ND; ++f) o[f] *= keep;
            m = next_m;
        }
        const float from = reference_of(m);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p[t][e] = exp2_of(fmaf(p[t][e], a.c, -from));
                l += p[t][e];
            }
        if (edge) {   // values behind the last key become 0; are the others finite?
            bool odd = false;
            auto check = [&](int L, u32x4_t w) {
                const int there = stop - (key + ((L % VP) ^ v_swap(L / VP)) * 8);
                w = Elem<uint16_t>::first_of(w, there);
                odd |= Elem<uint16_t>::not_finite(w);
                if (there < 8) *reinterpret_cast<u32x4_t *>(vt + L * 8) = w;
            };
            // With a window five steps of a tile's 19 come here (1024 keys, tiles of 32 tokens), so all pieces are asked for at once, and the next step's loads are not
            // waited for (two chunks of up to 2048 tokens: 114 us, 118 as below).  Elsewhere one or two do (16 trees of up to 26 tokens: 55.5 us, 54.3 - 55.3).
            if constexpr (WINDOW) {
                u32x4_t w[NV];
#pragma unroll
                for (int j = 0; j < NV; ++j) w[j] = *reinterpret_cast<const u32x4_t *>(vt + (tid + j * kAttnThreads) * 8);
#pragma unroll
                for (int j = 0; j < NV; ++j) check(tid + j * kAttnThreads, w[j]);
                if (odd) odd_seen = 1;
                lds_barrier();
                odd = __builtin_amdgcn_readfirstlane(odd_seen);
            } else {
#pragma unroll 1
                for (int L = tid; L < DP * VP; L += kAttnThreads) check(L, *reinterpret_cast<const u32x4_t *>(vt + L * 8));
                odd = __syncthreads_or(odd);
            }
            if (odd) {   // rare: what they add to the rows that see them, then 0 in their place
#pragma unroll 1
                for (int u = 0; u < 2 * TILES; ++u) {
                    const int c = (KW > 1 ? half * 4 : 0) + 2 * u + h;
                    const u32x4_t ones = Elem<uint16_t>::ones(seen(key + c * 8));
#pragma unroll
                    for (int f = 0; f < ND; ++f) {
                        const int d = f * 32 + n;
                        u32x4_t finite, kinds;
                        Elem<uint16_t>::part(*reinterpret_cast<const u32x4_t *>(vt + d * KEYS + (c ^ v_swap(d)) * 8), finite, kinds);
                        f32x16_t counts;
#pragma unroll
                        for (int e = 0; e < 16; ++e) counts[e] = 0.f;
                        counts = mma(kinds, ones, counts);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[f][e] += limit_of(counts[e]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __syncthreads();
                if (WINDOW && tid == 0) odd_seen = 0;   // read by all
#pragma unroll 1
                for (int L = tid; L < DP * VP; L += kAttnThreads) {
                    u32x4_t *at_piece = reinterpret_cast<u32x4_t *>(vt + L * 8);
                    *at_piece = Elem<uint16_t>::finite_of(*at_piece);
                }
                __syncthreads();
            }
        }
        // these products go before the softmax of the SIMD's other wave (64 drafted tokens on 131000 keys: 186 us, 191 without)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4_t pw;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pw[e] = two_bf16(p[t][8 * u + 2 * e], p[t][8 * u + 2 * e + 1]);
                    z = add_two_bf16(pw[e], z);
                }
                const int c = (KW > 1 ? half : t) * 4 + 2 * u + h;   // this lane's eight keys, as a piece of a row of V^T
#pragma unroll
                for (int f = 0; f < ND; ++f) {
                    const int d = f * 32 + n;
                    o[f] = mma(*reinterpret_cast<const u32x4_t *>(vt + d * KEYS + (c ^ v_swap(d)) * 8), pw, o[f]);
                }
            }
        __builtin_amdgcn_s_setprio(0);
    };

    if (WINDOW && tid == 0) odd_seen = 0;
    __syncthreads();
    const int steps = (stop - first + KEYS - 1) / KEYS;
    if (steps > 0) {
        request(0, k0, v0);
        __syncthreads();
        for (int i = 0;;) {
            if (i + 1 < steps) request(i + 1, k1, v1);
            compute(i, k0, v0);
            __syncthreads();   // everyone has read this step's tiles, the next ones have arrived
            if (++i >= steps) break;
            if (i + 1 < steps) request(i + 1, k0, v0);
            compute(i, k1, v1);
            __syncthreads();
            if (++i >= steps) break;
        }
    }

    {   // the other half of each row's keys that this wave takes lies in the lane 32 away
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(z), __float_as_uint(z), false, false);
        l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        z = __uint_as_float(u[0]) + __uint_as_float(u[1]);
    }
    if constexpr (KW > 1) {   // the second wave of a row group hands its sums to the first, lane for lane
        static_assert(KEYS * PITCH * 2 >= 32 * DP * 4, "a tile of K holds a wave's sums");
        f32x4_t *box = reinterpret_cast<f32x4_t *>(group ? k1 : k0);
        if (half == 1) {
#pragma unroll
            for (int f = 0; f < ND; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) box[(f * 4 + i) * kWave + lane] = f32x4_t{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]};
            if (h == 0) halves[group][n] = make_float4(m, l, z, 0.f);
        }
        __syncthreads();
        if (half == 1) return;
        const float4 other = halves[group][n];
        const float top = fmaxf(m, other.x), f0 = m == top ? 1.f : exp2_of(m - top), f1 = other.x == top ? 1.f : exp2_of(other.x - top);
        m = top;
        l = l * f0 + other.y * f1;
        z = z * f0 + other.z * f1;
#pragma unroll
        for (int f = 0; f < ND; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4_t x = box[(f * 4 + i) * kWave + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[f][4 * i + e] = o[f][4 * i + e] * f0 + x[e] * f1;
            }
    }
    if (row >= R) return;
#pragma unroll
    for (int f = 0; f < ND; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = f * 32 + 8 * i + 4 * h;
            if (EVEN || d < D) store_sums<uint16_t>(a, blk.chunk, at, d, f32x4_t{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]}, m, l, z);
        }
}

template <int DP, int RW, Kind KIND, bool EVEN>
void launch_tokens(const AttentionArgs &a, bool tokens, dim3 grid, hipStream_t stream) {
    if (tokens) hipLaunchKernelGGL((kv_rows_kernel<DP, RW, KIND, EVEN, true>), grid, dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv_rows_kernel<DP, RW, KIND, EVEN, false>), grid, dim3(kAttnThreads), 0, stream, a);
}

template <int DP, Kind KIND>
void launch_tiles(const AttentionArgs &a, int tiles, bool tokens, dim3 grid, hipStream_t stream) {
    if (tiles == 4) {
        if (a.p.dim == DP) launch_tokens<DP, 4, KIND, true>(a, tokens, grid, stream);
        else launch_tokens<DP, 4, KIND, false>(a, tokens, grid, stream);
    } else {
        if (a.p.dim == DP) launch_tokens<DP, 2, KIND, true>(a, tokens, grid, stream);
        else launch_tokens<DP, 2, KIND, false>(a, tokens, grid, stream);
    }
}

template <int DP>
void launch_dim(const AttentionArgs &a, Kind kind, int tiles, bool tokens, dim3 grid, hipStream_t stream) {
    if (kind == kWindow) launch_tiles<DP, kWindow>(a, tiles, tokens, grid, stream);
    else launch_tiles<DP, kAll>(a, tiles, tokens, grid, stream);
}

}  // namespace

void launch_kv_rows(const AttentionArgs &a, Kind kind, int tiles, bool tokens, dim3 grid, hipStream_t stream) {
    if (a.p.dim <= 64) launch_dim<64>(a, kind, tiles, tokens, grid, stream);
    else if (a.p.dim <= 96) launch_dim<96>(a, kind, tiles, tokens, grid, stream);
    else if (a.p.dim <= 128) launch_dim<128>(a, kind, tiles, tokens, grid, stream);
    else launch_dim<256>(a, kind, tiles, tokens, grid, stream);
}

}  // namespace tbn
