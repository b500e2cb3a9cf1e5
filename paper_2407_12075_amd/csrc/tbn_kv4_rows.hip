// Attention of many rows (drafted trees, prompt chunks; bfloat16) over the cache in 4 bits.  As in tbn_kv_rows.hip a workgroup takes 64 or 128 rows and
// goes through the keys 64 at a time, keys and values staged in LDS for all its waves, both products v_mfma_f32_32x32x16_bf16 with the query
// rows as columns.  Here the tiles are made: each thread takes its share of the codes and exponents of the step after next to registers, and, when this
// step's products are done, turns those of the next one into bfloat16 and stores them to the other buffer.
//
// So the conversion is paid once for all rows, and values, too, are multiplied by their powers of two there, pair by pair (two conversions with the two keys'
// scales, of which each gives one half): per row it would be the weights' (tbn_kv4_attention.hip), which costs 16 rows as much as this does 64.
//
// Values in LDS are finite whatever the cache holds (exponents are held within -126 .. 125): a weight of 0 leaves them out.
#include "tbn_kv4.h"
#include "tbn_kv_attention.h"

namespace tbn {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16_t mma(u32x4_t a, u32x4_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// The instruction's row of key r of a tile of 32, and the other way round: its output register 4 i + j of a lane of half h is row 8 i + 4 h + j, and a
// lane's eight logits in a row are to be of eight neighbouring keys.
__device__ __forceinline__ int row_of_key(int r) { return (r & 0x13) | (r & 4) << 1 | (r & 8) >> 1; }

template <int WORDS> struct Words { uint32_t w[WORDS]; };

// NB: groups of 32 channels.  RW: groups of 32 rows, 4 / RW waves each, which take alternate halves of the keys.  TOKENS: blockIdx.y is a token (sequence_of).
template <int NB, int RW, Kind KIND, bool TOKENS>
__global__ __launch_bounds__(kAttnThreads, NB <= 4 ? 2 : 1) void kv4_rows_kernel(AttentionArgs a) {
    constexpr bool WINDOW = KIND == kWindow;
    constexpr int KW = kAttnWaves / RW, KEYS = 64, TILES = 2 / KW;
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2, PITCH = (D + 63) / 64 * 64;   // PITCH: channels of a row of K in LDS
    __shared__ __attribute__((aligned(16))) uint16_t k0[KEYS * PITCH], k1[KEYS * PITCH], v0[D * KEYS], v1[D * KEYS];
    __shared__ int listed[kListed];
    __shared__ float4 halves[RW][32];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int s = sequence_of<TOKENS>(a);
    if (TOKENS && s < 0) return;
    const int H = a.q.heads, KV = a.p.kv_heads, G = H / KV, P = a.p.page, shift = __ffs(P) - 1, group = wave % RW, half = wave / RW;
    const Span v = span_of(a, s);
    const Block blk = block_of(a);
    const int R = v.T * G, base = blk.row_tile * (32 * RW);
    if (base >= R) return;
    const int last = min(base + 32 * RW, R) - 1;
    Within in_reach = {};
    if constexpr (WINDOW) in_reach = within_of(a, v, base, last, G, shift);
    const int end = WINDOW ? in_reach.end : keys_end(a, v, last, G);   // keys are counted along the pages that are gone through
    const int first = blk.chunk * a.chunk;
    if (first >= end && blk.chunk > 0) return;
    const int stop = min(end, first + a.chunk), entries = (stop - first + P - 1) >> shift;
    const int32_t *table = a.ix.table + int64_t(s) * a.ix.max_pages;
    for (int i = tid; i < entries; i += kAttnThreads)
        listed[i] = page_in(table[(WINDOW ? in_reach.key(first + (i << shift)) : first + (i << shift)) >> shift], static_cast<int>(a.p.n_pages));

    const int row = base + group * 32 + n, in = min(row, R - 1), place = in / G, low = WINDOW ? window_of(a, v, place) : 0;
    const int64_t at = int64_t(v.t0 + place) * H + blk.head * G + (in - place * G);   // of the outputs, where row < R
    u32x4_t q[NF];
    {
        const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (v.t0 + place) * a.q.q_stride + (blk.head * G + in - place * G) * D + 8 * h;
#pragma unroll
        for (int f = 0; f < NF; ++f) q[f] = *reinterpret_cast<const Elem<uint16_t>::u32x4_any *>(src + f * 16);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[f][e] = row < R ? q[f][e] ^ a.flip : 0u;
    }

    // This thread's share of a step: a quarter of the channels of one key; of eight keys (octet kg of a block of 32) the channels 16 f + kn, f from kf on.
    const int part = tid >> 7, key_row = (tid >> 2) & 31, quarter = tid & 3, kg = (tid >> 5) & 3, kn = (tid >> 1) & 15, kf = (tid & 1) * NB;
    struct Step {
        Words<NB> k, v;
        Words<EW> ke, ve[8];
    };
    const int64_t page_keys = int64_t(P) * KV;
    auto load = [&](Step &x, int i) {
        const int off = i * KEYS + part * 32, page = __builtin_amdgcn_readfirstlane(listed[min(off >> shift, entries - 1)]);
        const int64_t key = page * page_keys + int64_t(blk.head) * P + (off & (P - 1));
        x.k = *reinterpret_cast<const Words<NB> *>(static_cast<const uint32_t *>(a.p.k) + (key + key_row) * (D / 8) + quarter * NB);
        x.ke = *reinterpret_cast<const Words<EW> *>(a.p.summary + (key + key_row) * (4 * EW));
        x.v = *reinterpret_cast<const Words<NB> *>(static_cast<const uint32_t *>(a.p.v) + key * (D / 8) + (kg * 16 + kn) * NF + kf);
#pragma unroll
        for (int e = 0; e < 8; ++e) x.ve[e] = *reinterpret_cast<const Words<EW> *>(reinterpret_cast<const int8_t *>(a.p.step) + (key + 8 * kg + e) * (4 * EW));
    };
    auto store = [&](const Step &x, uint16_t *kt, uint16_t *vt) {
        const int r = part * 32 + row_of_key(key_row);
#pragma unroll
        for (int f = 0; f < NB; ++f) {
            const int c = (quarter * NB + f) >> 2;
            const uint32_t e = EW == 1 || c < 4 ? x.ke.w[0] : x.ke.w[EW - 1];
            *reinterpret_cast<u32x4_t *>(kt + r * PITCH + ((quarter * NB + f) ^ (r & 7)) * 8) = kv4_values(x.k.w[f], kv4_scale(e, c & 3));
        }
        const int piece = part * 4 + kg;
        float scale[8];
#pragma unroll
        for (int f = 0; f < NB; ++f) {
            const int c = (kf + f) >> 1;   // its group; words of one group lie side by side
            if (f == 0 || (NB & 1) || (f & 1) == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t word = EW == 1 || c < 4 ? x.ve[e].w[0] : x.ve[e].w[EW - 1];
                    const int y = min(max(static_cast<int>(static_cast<int8_t>(word >> (8 * (c & 3)))), -126), 125);
                    scale[e] = __uint_as_float(static_cast<uint32_t>(y + 127) << 23);
                }
            u32x4_t w;
            auto pair = [&](auto e) {
                const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.v.w[f], scale[2 * e()], e()));
                const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.v.w[f], scale[2 * e() + 1], e()));
                return (lo & 0xffffu) | (hi & 0xffff0000u);
            };
            w[0] = pair(std::integral_constant<int, 0>());
            w[1] = pair(std::integral_constant<int, 1>());
            w[2] = pair(std::integral_constant<int, 2>());
            w[3] = pair(std::integral_constant<int, 3>());
            const int d = 16 * (kf + f) + kn;
            *reinterpret_cast<u32x4_t *>(vt + d * KEYS + (piece ^ (d & 7)) * 8) = w;
        }
    };

    f32x16_t o[NB];
#pragma unroll
    for (int f = 0; f < NB; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[f][e] = 0.f;
    float m = -INFINITY, l = 0.f, z = 0.f;
    const int all_see = a.mask ? v.prefix : v.prefix + base / G + 1;   // keys from here on are not seen by every row
    const int all_from = WINDOW ? last_window(a, v, last, G) : 0;      // keys before this one, the first ones aside, neither

    auto compute = [&](int i, const uint16_t *kt, const uint16_t *vt) {
        f32x16_t p[2];   // of each tile, or two halves of the one tile's sum: chains of products that do not wait for each other
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) p[t][e] = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                p[TILES == 2 ? t : f & 1] = mma(*reinterpret_cast<const u32x4_t *>(kt + ((KW > 1 ? half : t) * 32 + n) * PITCH + ((2 * f + h) ^ (n & 7)) * 8), q[f], p[TILES == 2 ? t : f & 1]);
        if constexpr (TILES == 1) p[0] += p[1];
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
                    const int x = key + (KW > 1 ? half : t) * 32 + 16 * u + 8 * h, k = WINDOW ? in_reach.key(x) : x;
                    const uint32_t bits = seen_within<KIND>(a, v, k, stop + (k - x), place, low);
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
        if (__any(top > m)) {   // the reference is a little above the largest logit: weights are at most 1
            const float next_m = top > m ? top + kSlack : m, keep = next_m > m ? exp2_of(m - next_m) : 1.f;
            l *= keep;
            z *= keep;
#pragma unroll
            for (int f = 0; f < NB; ++f) o[f] *= keep;
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
                for (int f = 0; f < NB; ++f) {
                    const int d = f * 32 + n;
                    o[f] = mma(*reinterpret_cast<const u32x4_t *>(vt + d * KEYS + (c ^ (d & 7)) * 8), pw, o[f]);
                }
            }
        __builtin_amdgcn_s_setprio(0);
    };

    __syncthreads();
    const int steps = (stop - first + KEYS - 1) / KEYS;
    if (steps > 0) {
        Step x;
        load(x, 0);
        store(x, k0, v0);
        load(x, min(1, steps - 1));
        __syncthreads();
        for (int i = 0;;) {
            compute(i, k0, v0);
            store(x, k1, v1);   // behind the last step: nobody reads it
            load(x, min(i + 2, steps - 1));
            __syncthreads();   // everyone has read this step's tiles and stored the next one's
            if (++i >= steps) break;
            compute(i, k1, v1);
            store(x, k0, v0);
            load(x, min(i + 2, steps - 1));
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
        static_assert(KEYS * PITCH * 2 >= 32 * D * 4, "a tile of K holds a wave's sums");
        f32x4_t *box = reinterpret_cast<f32x4_t *>(group ? k1 : k0);
        if (half == 1) {
#pragma unroll
            for (int f = 0; f < NB; ++f)
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
        for (int f = 0; f < NB; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4_t x = box[(f * 4 + i) * kWave + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[f][4 * i + e] = o[f][4 * i + e] * f0 + x[e] * f1;
            }
    }
    if (row >= R) return;
#pragma unroll
    for (int f = 0; f < NB; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_sums<uint16_t>(a, blk.chunk, at, f * 32 + 8 * i + 4 * h, f32x4_t{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]}, m, l, z);
}

template <int NB, int RW, Kind KIND>
void launch_tokens(const AttentionArgs &a, bool tokens, dim3 grid, hipStream_t stream) {
    if (tokens) hipLaunchKernelGGL((kv4_rows_kernel<NB, RW, KIND, true>), grid, dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv4_rows_kernel<NB, RW, KIND, false>), grid, dim3(kAttnThreads), 0, stream, a);
}

}  // namespace

void launch_kv4_rows(const AttentionArgs &a, Kind kind, int tiles, bool tokens, dim3 grid, hipStream_t stream) {
    kv4_by_groups(a.p.dim, [&](auto nb) {
        if (kind == kWindow) {
            if (tiles == 4) launch_tokens<nb(), 4, kWindow>(a, tokens, grid, stream);
            else launch_tokens<nb(), 2, kWindow>(a, tokens, grid, stream);
        } else {
            if (tiles == 4) launch_tokens<nb(), 4, kAll>(a, tokens, grid, stream);
            else launch_tokens<nb(), 2, kAll>(a, tokens, grid, stream);
        }
    });
}

}  // namespace tbn
