// Attention over a cache held in 4 bits.  Mathematics, masks, windows and parts as in tbn_kv_attention.hip; the cache's bytes are about a quarter
// of bfloat16's, so what the vector units do for each key counts as much as what comes from memory.
//
//   S^T = K Q^T,  O^T += V^T P^T  (v_mfma_f32_16x16x32_bf16, keys or channels as rows, query rows as columns)
//
// A workgroup takes 16 rows, or (FEW) as many as leave each of the 16 columns a row and a group of channels; its waves take steps of 32 keys in turn.
// A lane loads a quarter of a key's channels (dim / 8 bytes: 16 of 128 channels) of two keys, and eight keys of dim / 16 channels (dim / 4 bytes in a row,
// the order of the cache).  The order in which the first product goes through the channels is free, so a lane's quarter is one run of them and q
// is loaded to match.
//
// A key's numbers are codes times 2^x, x for 32 channels.  Keys: the conversion to bfloat16 multiplies, which is exact.  Values: eight keys in a
// lane's word have eight exponents, so they go to the weights instead: p 2^x is rounded to bfloat16 once for each 32 channels, with p's own
// relative error, and the codes are taken as they are.  FEW, decoding above all: a column of P^T is a row's weights for one group, so that a lane makes them
// once, not for each group, and of the second product each group's channels are taken from its own columns.  Codes are always finite: a
// weight of 0 is enough to leave a value out.  A key that is no number gives not-a-number logits, and its row is that all over.
//
// float32 queries: q is the sum of three bfloat16 numbers (8 bits each), exactly, and so is each weight to 2^-24: three products of each kind.
#include "tbn_kv4.h"
#include "tbn_kv_attention.h"

namespace tbn {

namespace {

__device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Two numbers as sums of bfloat16 ones: what is left of them after each
__device__ __forceinline__ uint32_t split_off(float &lo, float &hi) {
    const uint32_t pair = two_bf16(lo, hi);
    lo -= __uint_as_float(pair << 16);
    hi -= __uint_as_float(pair & 0xffff0000u);
    return pair;
}

template <typename T> struct Query;
template <> struct Query<uint16_t> {
    static constexpr int kTerms = 1;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ void load(const uint16_t *at, uint32_t flip, bool there, u32x4_t (&q)[1]) {
        const u32x4_t w = *reinterpret_cast<const any *>(at);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[0][e] = there ? w[e] ^ flip : 0u;
    }
};
template <> struct Query<float> {
    static constexpr int kTerms = 3;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void load(const float *at, uint32_t flip, bool there, u32x4_t (&q)[3]) {
        const u32x4_t w[2] = {*reinterpret_cast<const any *>(at), *reinterpret_cast<const any *>(at + 4)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float lo = __uint_as_float(there ? w[e / 2][2 * (e & 1)] ^ flip : 0u), hi = __uint_as_float(there ? w[e / 2][2 * (e & 1) + 1] ^ flip : 0u);
            // The first terms are cut, not rounded: the nearest bfloat16 to the largest numbers is infinite, and the 16 bits left fill two more.  A number that
            // is not finite stays what it is in the first term (less itself it would be none in the others).
            const bool fl = fabsf(lo) < INFINITY, fh = fabsf(hi) < INFINITY;
            const uint32_t first = two_bf16(lo, hi);
            const uint32_t l = fl ? __float_as_uint(lo) >> 16 : first & 0xffffu, h = fh ? __float_as_uint(hi) & 0xffff0000u : first & 0xffff0000u;
            q[0][e] = l | h;
            lo = fl ? lo - __uint_as_float(l << 16) : 0.f;
            hi = fh ? hi - __uint_as_float(h) : 0.f;
            q[1][e] = split_off(lo, hi);
            q[2][e] = split_off(lo, hi);
        }
    }
};

template <int WORDS> struct Words { uint32_t w[WORDS]; };

// Rows of a workgroup whose lanes share the groups of channels: each of the product's 16 columns is a row and a group.
constexpr int shared_rows(int nb) { return nb == 1 ? 16 : nb == 2 ? 8 : nb <= 4 ? 4 : 2; }

// Workgroups of a CU, by the registers that one takes.  Three are enough: 64 sequences of 4096 - 16384 keys take as long with four (151 us; a streaming
// read of their bytes 135) and, where registers would have to be spilled for that, longer.
constexpr int workgroups_of(int nb, int size) { return size == 2 ? (nb <= 4 ? 3 : nb == 5 ? 2 : 1) : nb <= 2 ? 3 : nb <= 4 ? 2 : 1; }

// NB: groups of 32 channels.  FEW: at most shared_rows(NB) rows; TOKENS: blockIdx.y is a token (sequence_of).
template <int NB, typename T, Kind KIND, bool FEW, bool TOKENS>
__global__ __launch_bounds__(kAttnThreads, workgroups_of(NB, sizeof(T))) void kv4_attention_kernel(AttentionArgs a) {
    constexpr bool WINDOW = KIND == kWindow;
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2, TERMS = Query<T>::kTerms, KS = 32;
    constexpr int ROWS = FEW ? shared_rows(NB) : 16, NC = FEW ? 1 : NB;   // NC: groups that a lane's weights are made for
    __shared__ int2 listed[kListed];   // slot and page
    __shared__ float sums[kAttnWaves][ROWS][D + 4];
    __shared__ float maxima[kAttnWaves][ROWS], totals[2][kAttnWaves][ROWS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int col = n & (ROWS - 1), own = FEW ? n / ROWS : 0;   // this lane's row and, FEW, group of channels
    const int s = sequence_of<TOKENS>(a);
    if (TOKENS && s < 0) return;
    const int H = a.q.heads, KV = a.p.kv_heads, G = H / KV, P = a.p.page, shift = __ffs(P) - 1;
    const Span v = span_of(a, s);
    const Block blk = block_of(a);
    const int head = blk.head, chunk = blk.chunk, base = blk.row_tile * ROWS, R = v.T * G;
    if (base >= R) return;
    const int last = min(base + ROWS, R) - 1, end = keys_end(a, v, last, G);
    Within in_reach = {};
    if constexpr (WINDOW) in_reach = within_of(a, v, base, last, G, shift);
    const int first = chunk * a.chunk, stop = WINDOW ? in_reach.end : end;
    if (first >= stop && chunk > 0) return;
    const int entries = (min(stop, first + a.chunk) - first + P - 1) >> shift;
    const int32_t *table = a.ix.table + int64_t(s) * a.ix.max_pages;
    for (int i = tid; i < entries; i += kAttnThreads) {
        const int slot = (WINDOW ? in_reach.key(first + (i << shift)) : first + (i << shift)) >> shift;
        listed[i] = make_int2(slot, page_in(table[slot], static_cast<int>(a.p.n_pages)));
    }

    const int row = base + col, place = min(row, R - 1) / G, low = WINDOW ? window_of(a, v, place) : 0;
    u32x4_t q[NB][TERMS];
    {
        const T *src = static_cast<const T *>(a.q.q) + (v.t0 + place) * a.q.q_stride + (head * G + min(row, R - 1) - place * G) * D + g * (8 * NB);
#pragma unroll
        for (int f = 0; f < NB; ++f) Query<T>::load(src + 8 * f, a.flip, row < R, q[f]);
    }

    f32x4_t o[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f, z = 0.f;   // reference, sum of the weights, of the rounded weights (float32: the same, not kept)

    // what a step takes from the cache: codes and exponents of two keys (rows n of the product's two tiles) and of eight keys' values
    struct Step {
        Words<NB> k[2];
        Words<EW> ke[2];
        Words<NF> v;
        Words<EW> ve[8];
    };
    const int k_key = 8 * (n >> 2) + (n & 3);   // of the first tile, + 4 in the second: a lane's eight logits are of keys 8 g .. 8 g + 7
    const int64_t page_keys = int64_t(P) * KV;
    auto load_k = [&](Step &x, int page, int off) {
        const int64_t key = page * page_keys + int64_t(head) * P + off + k_key;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            x.k[t] = *reinterpret_cast<const Words<NB> *>(static_cast<const uint32_t *>(a.p.k) + (key + 4 * t) * (D / 8) + g * NB);
            x.ke[t] = *reinterpret_cast<const Words<EW> *>(a.p.summary + (key + 4 * t) * (4 * EW));
        }
    };
    auto load_v = [&](Step &x, int page, int off) {
        const int64_t key = page * page_keys + int64_t(head) * P + off;
        x.v = *reinterpret_cast<const Words<NF> *>(static_cast<const uint32_t *>(a.p.v) + key * (D / 8) + (g * 16 + n) * NF);
#pragma unroll
        for (int e = 0; e < 8; ++e) x.ve[e] = *reinterpret_cast<const Words<EW> *>(reinterpret_cast<const int8_t *>(a.p.step) + (key + 8 * g + e) * (4 * EW));
    };
    const int sub_shift = shift - 5, steps = entries << sub_shift;
    // step i of this stretch: its first key, -1 if there is nothing in it; wave-uniform
    auto key_of = [&](int i, int &page) {
        const int2 e = listed[i >> sub_shift];
        page = __builtin_amdgcn_readfirstlane(e.y);
        const int key = (__builtin_amdgcn_readfirstlane(e.x) << shift) + (i & ((1 << sub_shift) - 1)) * KS;
        if (WINDOW && key >= a.window.sink && key + KS <= in_reach.low) return -1;
        return key >= end ? -1 : key;
    };
    auto next_step = [&](int i, int &key, int &page) {
        while (i < steps) {
            key = key_of(i, page);
            if (key >= 0) break;
            i += kAttnWaves;
        }
        return i;
    };

    const int all_see = a.mask ? v.prefix : v.prefix + base / G + 1;   // keys from here on are not seen by every row
    const int all_from = WINDOW ? last_window(a, v, last, G) : 0;      // keys before this one, the first ones aside, neither
    __syncthreads();
    Step x;
    int key = 0, page = 0;
    int i = next_step(wave, key, page);
    if (i < steps) {
        load_k(x, page, key & (P - 1));
        load_v(x, page, key & (P - 1));
    }
    while (i < steps) {
        float p[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                const int c = (g * NB + f) >> 2;   // the group that these eight channels lie in
                const uint32_t e = EW == 1 ? x.ke[h].w[0] : c < 4 ? x.ke[h].w[0] : x.ke[h].w[EW - 1];
                const u32x4_t k = kv4_values(x.k[h].w[f], kv4_scale(e, c & 3));
                if constexpr (TERMS == 3) {
                    s1 = mma(k, q[f][2], s1);
                    s1 = mma(k, q[f][1], s1);
                }
                s0 = mma(k, q[f][0], s0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)   // an infinite logit is one already in the first terms, whatever the others' signs
                p[4 * h + e] = TERMS == 3 && fabsf(s0[e]) < INFINITY ? s0[e] + s1[e] : s0[e];
        }
        // the next step's loads, or the same ones again: never left out, so that the waits before their use are for as many as there are
        int next_key = 0, next_page = 0;
        const int next = next_step(i + kAttnWaves, next_key, next_page);
        if (next >= steps) {
            next_key = key;
            next_page = page;
        }
        load_k(x, next_page, next_key & (P - 1));

        bool edge = key + KS > all_see;   // wave-uniform
        if constexpr (WINDOW) edge |= key < all_from && key + KS > a.window.sink;
        if (edge) {
            const uint32_t bits = seen_within<KIND>(a, v, key + 8 * g, end, place, low);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = (bits >> e) & 1u ? p[e] : -INFINITY;
        }
        float top = p[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, p[e]);
        top = max_over_32(max_over_16(top)) * a.c;
        if (__any(top > m)) {   // the reference is a little above the largest logit: weights are at most 1, so that p 2^x does not leave the range of numbers
            const float next_m = top > m ? top + kSlack : m, keep = next_m > m ? exp2_of(m - next_m) : 1.f;   // the first time 2^-inf = 0
            l *= keep;
            z *= keep;
#pragma unroll
            for (int f = 0; f < NF; ++f) o[f] *= keep;
            m = next_m;
        }
        const float from = reference_of(m);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = exp2_of(fmaf(p[e], a.c, -from));
            l += p[e];
        }
        if constexpr (TERMS == 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) z = add_two_bf16(two_bf16(p[2 * e], p[2 * e + 1]), z);
        u32x4_t w[NC][TERMS];   // the weights as operand, times the values' powers of two
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                auto times = [&](int j) {
                    const int b = FEW ? own : c;
                    const uint32_t word = EW == 1 || b < 4 ? x.ve[j].w[0] : x.ve[j].w[EW - 1];
                    return __builtin_ldexpf(p[j], static_cast<int8_t>(word >> (8 * (b & 3))));
                };
                float lo = times(2 * e), hi = times(2 * e + 1);
                if constexpr (TERMS == 1) w[c][0][e] = two_bf16(lo, hi);
                else
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) w[c][t][e] = split_off(lo, hi);
            }
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const u32x4_t d = kv4_values(x.v.w[f], 1.f);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) o[f] = mma(d, w[FEW ? 0 : f / 2][t], o[f]);
        }
        load_v(x, next_page, next_key & (P - 1));
        i = next;
        key = next_key;
        page = next_page;
    }

    // the waves' sums
    float ls = l, zs = TERMS == 1 ? z : l;
    ls += __shfl_xor(ls, 16);
    ls += __shfl_xor(ls, 32);
    zs += __shfl_xor(zs, 16);
    zs += __shfl_xor(zs, 32);
    if (lane < ROWS) {
        maxima[wave][lane] = m;
        totals[0][wave][lane] = ls;
        totals[1][wave][lane] = zs;
    }
    __syncthreads();
    float top = maxima[0][col];
#pragma unroll
    for (int u = 1; u < kAttnWaves; ++u) top = fmaxf(top, maxima[u][col]);
    const float f0 = m == top ? 1.f : exp2_of(m - top);
#pragma unroll
    for (int f = 0; f < NF; ++f)
        if (!FEW || own == f / 2) *reinterpret_cast<f32x4_t *>(&sums[wave][col][f * 16 + 4 * g]) = o[f] * f0;
    __syncthreads();
    for (int j = tid; j < ROWS * (D / 4); j += kAttnThreads) {
        const int rr = j / (D / 4), d = (j - rr * (D / 4)) * 4, row = base + rr;
        if (row >= R) continue;
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
            sum += *reinterpret_cast<const f32x4_t *>(&sums[u][rr][d]);
        }
        const int t = row / G;
        store_sums<T>(a, chunk, int64_t(v.t0 + t) * H + head * G + row - t * G, d, sum, best, lsum, zsum);
    }
}

// The queries' view of the cache: sizes as there, the queries' type.
tbn_kv_pool view_of(const tbn_kv4_pool &p, tbn_dtype dt) { return tbn_kv_pool{p.k, p.v, p.k_exp, reinterpret_cast<float *>(p.v_exp), p.n_pages, p.kv_heads, p.dim, p.page, dt}; }

Plan plan_of(const tbn_kv_pool &p, int64_t rows, int64_t groups, int64_t keys, bool window) {
    Plan pl;
    const int few = shared_rows(p.dim / 32);
    // The kernel that stages keys takes as long for 64 (128) rows as this file's for about 4 (7) tiles of 16, whose last ones ragged drafts often do not
    // need.  16 trees of up to 16 / 24 / 26 / 32 tokens on 4000 keys, 4 heads to a kv head: 40 / 51 / 54 / 55 us, here 44 / 49 / 47 / 65; 12 tokens 38 to 33.  On many
    // keys it is the faster one with fewer (26 tokens on 60000 keys: 56 us, 77 here; 10 tokens level); 512 tokens on 16000: 173 us to 292.
    pl.staged = p.dt == TBN_BF16 && rows > 48 && (rows <= 64 || rows > 112 || keys >= 16384);
    const int64_t places = p.dim <= 128 ? 512 : 256;   // for workgroups of the kernel that stages keys
    pl.rows = pl.staged ? (rows <= 64 || (window && rows_of_64(rows, groups, keys, places)) ? 64 : 128) : rows <= few ? few : 16;
    pl.row_tiles = static_cast<int>(ceil_div(rows, pl.rows));
    const int64_t blocks = groups * pl.row_tiles;
    int64_t chunk;
    if (pl.staged) {
        // one round of the places for workgroups (512 tokens on 16000 keys: 173 us, 183 in two, 191 in four)
        chunk = std::max<int64_t>(std::min<int64_t>(256, keys), ceil_div(keys, ceil_div(places, blocks)));
        if (window && keys <= kFewKeys && blocks >= places / 2) chunk = keys;   // 1024 tokens, window 1024: 43 us, 54 in parts
    } else {
        // fill: keys of each place for a workgroup.  Up to 1024 one round of the places, 256 keys at least (bfloat16, 128 channels, 8 kv heads: 16 sequences of
        // 3000 keys 15.6 us with 512, 17.6 with 384, 18.5 with 256; one of 8000 keys 10.3 with 256, 12.5 with 128; one of 60000 keys 20 - 21 with 768 - 1024, 23.6 with 384).
        // Beyond, several stretches a place even out ragged sequences, against what starting each costs: 15 sqrt(fill), up to 1536 (64 sequences of up to
        // 16384 keys: 151 us; 154 with 1152, 160 with 2304, 180 with 512).
        const double fill = static_cast<double>(keys) * blocks / (256 * workgroups_of(p.dim / 32, p.dt == TBN_F32 ? 4 : 2));
        const double want = fill <= 1024 ? std::fmax(256, fill) : std::fmin(1536, 15 * std::sqrt(fill));
        chunk = std::max(ceil_div(keys, ceil_div(8192, blocks)), fill <= 1024 ? static_cast<int64_t>(std::ceil(want / 128)) * 128 : static_cast<int64_t>(want / 128 + 0.5) * 128);
        if (keys <= 1024 && blocks >= 256) chunk = keys;   // the join would take longer
    }
    // nor are few keys split, where the join's launch takes longer than the steps it saves (one token, 8 kv heads of 128 channels: 513 keys 7.3 us, 10.7 in
    // parts; 1000 keys 9.2 to 9.7, 1500 11.8 to 10.1; float32 513 keys 9.5 to 10.1, 1000 12.2 to 10.1)
    if (!pl.staged && keys <= (p.dt == TBN_BF16 ? 1024 : 640)) chunk = keys;
    chunk = ceil_div(keys, ceil_div(keys, chunk));   // of one length (64 sequences of 2000 keys, float32: 47 us, 52 with a short last one)
    chunk = std::min(ceil_div(chunk, 128) * 128, int64_t(kListed) * p.page);
    pl.chunk = static_cast<int>(chunk);
    pl.n_chunks = static_cast<int>(ceil_div(keys, chunk));
    return pl;
}

Plan plan_of_call(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_sink, int32_t window, bool masked) {
    const int64_t keys = window ? window_keys(p, q, n_sink, window, masked) : q.max_len;
    return plan_by_sequences(p, ix, q, keys, [&](int64_t rows, int64_t groups, int64_t units) { return plan_of(p, rows, groups, units, window != 0); });
}

template <int NB, typename T, Kind KIND, bool FEW>
void launch_tokens(const AttentionArgs &a, bool tokens, dim3 grid, hipStream_t stream) {
    if (tokens) hipLaunchKernelGGL((kv4_attention_kernel<NB, T, KIND, FEW, true>), grid, dim3(kAttnThreads), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attention_kernel<NB, T, KIND, FEW, false>), grid, dim3(kAttnThreads), 0, stream, a);
}

template <int NB, typename T, Kind KIND>
void launch_rows(const AttentionArgs &a, int rows, bool tokens, dim3 grid, hipStream_t stream) {
    if constexpr (NB > 1) {
        if (rows < 16) return launch_tokens<NB, T, KIND, true>(a, tokens, grid, stream);
    }
    launch_tokens<NB, T, KIND, false>(a, tokens, grid, stream);
}

template <int NB>
void launch_groups(const AttentionArgs &a, Kind kind, int rows, bool tokens, dim3 grid, hipStream_t stream) {
    if (a.p.dt == TBN_F32) {
        if (kind == kWindow) launch_rows<NB, float, kWindow>(a, rows, tokens, grid, stream);
        else launch_rows<NB, float, kAll>(a, rows, tokens, grid, stream);
    } else {
        if (kind == kWindow) launch_rows<NB, uint16_t, kWindow>(a, rows, tokens, grid, stream);
        else launch_rows<NB, uint16_t, kAll>(a, rows, tokens, grid, stream);
    }
}

}  // namespace

size_t kv4_attention_workspace(const tbn_kv4_pool &pool, const tbn_kv_index &ix, const KvQueries &q, tbn_dtype dt, int32_t n_sink, int32_t window, bool masked) {
    const tbn_kv_pool p = view_of(pool, dt);
    return workspace_of(p, q, plan_of_call(p, ix, q, n_sink, window, masked));
}

tbn_status launch_kv4_attention(const tbn_kv4_pool &pool, const tbn_kv_index &ix, const KvQueries &q, tbn_dtype dt, void *out, float *lse, int32_t n_sink,
                                int32_t window, const uint32_t *mask, int32_t mask_words, float scale, float *ws, hipStream_t stream) {
    const char *what = "tbn_kv4_attention";
    const Kind kind = window ? kWindow : kAll;
    const tbn_kv_pool p = view_of(pool, dt);
    AttentionArgs a{p, ix, q, out, lse, mask, mask_words, {nullptr}, 0, factor_of(scale), flip_of(p, scale)};
    a.window.sink = n_sink;
    a.window.size = window;
    const Plan pl = plan_of_call(p, ix, q, n_sink, window, mask != nullptr);
    dim3 grid;
    bool tokens;
    const tbn_status st = spread(a, pl, ws, kind, what, grid, tokens);
    if (st != TBN_OK) return st;
    if (pl.staged) launch_kv4_rows(a, kind, pl.rows / 32, tokens, grid, stream);
    else kv4_by_groups(p.dim, [&](auto nb) { launch_groups<nb()>(a, kind, pl.rows, tokens, grid, stream); });
    if (a.n_chunks > 1) launch_kv_join(a, kind, pl.rows, tokens, grid.y, stream);
    return check_launch(what);
}

}  // namespace tbn
