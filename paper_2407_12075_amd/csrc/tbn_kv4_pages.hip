// The cache held in 4 bits: new keys enter it, are read back, move between pages and within a sequence.
//
// A group is 32 channels of a key (a value) of one head: x the least whole number with max |.| <= 6 * 2^x, codes the nearest of
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times 2^x, by the hardware's conversion (nearest even, saturating).  Keys lie as rows.  Values lie in blocks of
// 32 keys as words of eight keys of a channel, in the order in which the attention's matrix instruction takes them:
//
//   word [g][n][f] of a block: keys 8 g .. 8 g + 7, channel 16 f + n, f < dim / 16; key 8 g + e in bits 4 e .. 4 e + 3
//
// so a key that enters a word others have is put between their bits.  One wave takes a block of a head; no two of a launch write to one word.
//
// Everything here moves bytes.
#include "tbn_kv4.h"

namespace tbn {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;   // keys

template <typename T> struct Eight;   // elements in a row, at any address that holds elements
template <> struct Eight<uint16_t> {
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ void load(const uint16_t *at, float (&f)[8]) {
        const u32x4_t w = *reinterpret_cast<const any *>(at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(uint16_t *at, u32x4_t w) { *reinterpret_cast<any *>(at) = w; }
};
template <> struct Eight<float> {
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void load(const float *at, float (&f)[8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4_t w = *reinterpret_cast<const any *>(at + 4 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[4 * h + i] = __uint_as_float(w[i]);
        }
    }
    static __device__ __forceinline__ void store(float *at, u32x4_t w) {   // of bfloat16 pairs
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<any *>(at + 4 * h) = u32x4_t{w[2 * h] << 16, w[2 * h] & 0xffff0000u, w[2 * h + 1] << 16, w[2 * h + 1] & 0xffff0000u};
    }
};

// the largest of four neighbouring lanes' values
__device__ __forceinline__ float max_of_quad(float a) {
    a = fmaxf(a, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), 0xb1, 0xf, 0xf, true)));
    return fmaxf(a, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(a), 0x4e, 0xf, 0xf, true)));
}

// A wave's share of the last n keys of a sequence: rows [r0, r1) of a block of 32 of one head, from token `tok` of the call on.
struct Share {
    int64_t page;      // pages before it, times heads: the (page, head) that the block lies in
    int block, r0, r1, tok;
};

__device__ __forceinline__ bool share_of(const tbn_kv4_pool &p, const tbn_kv_index &ix, const int32_t *cu, int total, Share &sh) {
    const int s = blockIdx.z, shift = __ffs(p.page) - 1;
    int t0;
    const int n = tokens_in(cu, s, total, t0), len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift);
    if (n <= 0 || n > len) return false;
    const int base = ((len - n) & -kBlock) + static_cast<int>(blockIdx.x) * kBlock;
    if (base >= len) return false;
    sh.page = int64_t(page_in(ix.table[int64_t(s) * ix.max_pages + (base >> shift)], static_cast<int>(p.n_pages))) * p.kv_heads + blockIdx.y;
    sh.block = (base & (p.page - 1)) / kBlock;
    sh.r0 = max(len - n - base, 0);
    sh.r1 = min(len - base, kBlock);
    sh.tok = t0 + base + sh.r0 - (len - n);
    return true;
}

// NB: groups of 32 channels of a head
template <typename T, int NB>
__global__ __launch_bounds__(kWave) void kv4_append_kernel(tbn_kv4_pool p, tbn_kv_index ix, const T *__restrict__ k_new, int64_t k_stride,
                                                           const T *__restrict__ v_new, int64_t v_stride, const int32_t *__restrict__ cu_new, int total) {
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2, PITCH = 40;   // EW: words of exponents of a key; PITCH: bytes of a channel in LDS
    __shared__ __attribute__((aligned(8))) uint8_t codes[D * PITCH];
    __shared__ uint32_t exps[2][kBlock][EW];
    __shared__ int odd[kBlock];
    const int lane = threadIdx.x;
    Share sh;
    if (*ix.status || !share_of(p, ix, cu_new, total, sh)) return;
    const int rows = sh.r1 - sh.r0;
    const T *ks = k_new + sh.tok * k_stride + blockIdx.y * D, *vs = v_new + sh.tok * v_stride + blockIdx.y * D;
    const int64_t first = sh.page * p.page + sh.block * kBlock + sh.r0;   // key of this layer that row r0 is
    uint32_t *kc = static_cast<uint32_t *>(p.k) + first * (D / 8), *vc = static_cast<uint32_t *>(p.v) + (sh.page * p.page + sh.block * kBlock) * (D / 8);
    if (lane < kBlock) odd[lane] = 0;
    for (int i = lane; i < 2 * kBlock * EW; i += kWave) exps[i / (kBlock * EW)][i / EW % kBlock][i % EW] = 0;
    __syncthreads();
    int8_t *x8 = reinterpret_cast<int8_t *>(exps);
    // Eight channels of a key, then of a value.  kAhead rounds are loaded before the first is looked at; lanes behind the last one take it again, so
    // that all go through the exchange between lanes together, and write nothing.
    constexpr int kAhead = 4;
    const int units = 2 * rows * 4 * NB;
    for (int i0 = lane; i0 - lane < units; i0 += kAhead * kWave) {
        float f[kAhead][8];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int i = min(i0 + j * kWave, units - 1), r = i / (4 * NB), c = i - r * (4 * NB);
            Eight<T>::load(r >= rows ? vs + (r - rows) * v_stride + 8 * c : ks + r * k_stride + 8 * c, f[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 - lane + j * kWave >= units) break;
            const int i = min(i0 + j * kWave, units - 1), r = i / (4 * NB), c = i - r * (4 * NB);
            const bool value = r >= rows;
            const int at = value ? r - rows : r;
            float a = 0.f;
            bool bad = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a = fmaxf(a, fabsf(f[j][e]));
                bad |= !(fabsf(f[j][e]) < INFINITY);
            }
            const int x = kv4_exponent(max_of_quad(a));
            if (i0 + j * kWave >= units) continue;
            const uint32_t w = kv4_codes(f[j], pow2_of(x));
            if (value) {
                uint8_t *to = codes + 8 * c * PITCH + sh.r0 + at;
#pragma unroll
                for (int e = 0; e < 8; ++e) to[e * PITCH] = (w >> (4 * e)) & 15u;
            } else {
                kc[at * (D / 8) + c] = w;
            }
            if ((c & 3) == 0) x8[((value ? kBlock : 0) + at) * (4 * EW) + (c >> 2)] = static_cast<int8_t>(x);
            if (bad) odd[at] = 1;
        }
    }
    __syncthreads();
    for (int i = lane; i < 2 * rows * EW; i += kWave) {
        const int r = i / EW, at = r >= rows ? r - rows : r;
        const uint32_t w = odd[at] ? 0x80808080u : exps[r >= rows][at][i % EW];
        reinterpret_cast<uint32_t *>(r >= rows ? p.v_exp : p.k_exp)[(first + at) * EW + i % EW] = w;
    }
    const int g0 = sh.r0 >> 3, octets = ((sh.r1 + 7) >> 3) - g0;
#pragma unroll 2
    for (int i = lane; i < octets * 16 * NF; i += kWave) {
        const int g = g0 + i / (16 * NF), j = i % (16 * NF), d = 16 * (j % NF) + j / NF;
        const uint32_t w = kv4_pack(*reinterpret_cast<const uint2 *>(codes + d * PITCH + 8 * g));
        const int lo = max(sh.r0 - 8 * g, 0), hi = min(sh.r1 - 8 * g, 8);
        const uint32_t mine = (hi == 8 ? ~0u : (1u << (4 * hi)) - 1u) & (~0u << (4 * lo));
        uint32_t *to = vc + g * 16 * NF + j;
        *to = mine == ~0u ? w : (*to & ~mine) | (w & mine);
    }
}

template <typename T, int NB>
__global__ __launch_bounds__(kWave) void kv4_read_kernel(tbn_kv4_pool p, tbn_kv_index ix, T *__restrict__ k_out, T *__restrict__ v_out,
                                                         const int32_t *__restrict__ cu, int total) {
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2, PITCH = D + 8;
    __shared__ __attribute__((aligned(8))) uint8_t codes[kBlock * PITCH];
    const int lane = threadIdx.x;
    Share sh;
    if (!share_of(p, ix, cu, total, sh)) return;
    const int rows = sh.r1 - sh.r0;
    const int64_t first = sh.page * p.page + sh.block * kBlock + sh.r0, row = int64_t(p.kv_heads) * D, to = sh.tok * row + blockIdx.y * D;
    const uint32_t *kc = static_cast<const uint32_t *>(p.k) + first * (D / 8), *vc = static_cast<const uint32_t *>(p.v) + (sh.page * p.page + sh.block * kBlock) * (D / 8);
    const int g0 = sh.r0 >> 3, octets = ((sh.r1 + 7) >> 3) - g0;
#pragma unroll 2
    for (int i = lane; i < octets * 16 * NF; i += kWave) {
        const int g = g0 + i / (16 * NF), j = i % (16 * NF), d = 16 * (j % NF) + j / NF;
        const uint32_t w = vc[g * 16 * NF + j];
#pragma unroll
        for (int e = 0; e < 8; ++e) codes[(8 * g + e) * PITCH + d] = (w >> (4 * e)) & 15u;
    }
    __syncthreads();
#pragma unroll 4
    for (int i = lane; i < 2 * rows * 4 * NB; i += kWave) {
        const int r = i / (4 * NB), c = i - r * (4 * NB);
        const bool value = r >= rows;
        const int at = value ? r - rows : r;
        const uint32_t x = reinterpret_cast<const uint32_t *>(value ? p.v_exp : p.k_exp)[(first + at) * EW + (c >> 4)];
        const uint32_t w = value ? kv4_pack(*reinterpret_cast<const uint2 *>(codes + (sh.r0 + at) * PITCH + 8 * c)) : kc[at * (D / 8) + c];
        Eight<T>::store((value ? v_out : k_out) + to + at * row + 8 * c, kv4_values(w, kv4_scale(x, (c >> 2) & 3)));
    }
}

constexpr int kPiece = 8192;   // bytes that a workgroup copies at a time

__global__ __launch_bounds__(256) void kv4_copy_kernel(tbn_kv4_pool p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int64_t n,
                                                       const int32_t *__restrict__ count, int code_bytes, int exp_bytes) {
    if (count) n = min(n, static_cast<int64_t>(max(*count, 0)));
    const int code_pieces = (code_bytes + kPiece - 1) / kPiece, exp_pieces = (exp_bytes + kPiece - 1) / kPiece, per = 2 * (code_pieces + exp_pieces);
    for (int64_t item = blockIdx.x; item < n * per; item += gridDim.x) {
        const int64_t pair = item / per;
        int what = static_cast<int>(item - pair * per);
        const int a = src[pair], b = dst[pair];
        if (a < 0 || b < 0 || a >= p.n_pages || b >= p.n_pages) continue;
        const bool exps = what >= 2 * code_pieces;
        what -= exps ? 2 * code_pieces : 0;
        const int pieces = exps ? exp_pieces : code_pieces, bytes = exps ? exp_bytes : code_bytes;
        const bool value = what >= pieces;
        const int at = (value ? what - pieces : what) * kPiece, end = min(kPiece, bytes - at);
        char *base = exps ? reinterpret_cast<char *>(value ? p.v_exp : p.k_exp) : static_cast<char *>(value ? p.v : p.k);
        const char *from = base + int64_t(a) * bytes + at;
        char *to = base + int64_t(b) * bytes + at;
        for (int o = threadIdx.x * 16; o < end; o += 256 * 16) *reinterpret_cast<u32x4_t *>(to + o) = *reinterpret_cast<const u32x4_t *>(from + o);
    }
}

constexpr int kThreads = 256;

// A workgroup takes a head of a sequence, 32 keys between their loads and their stores.  Picks ascend and are at or above their places, so a
// round's sources lie behind every target of the rounds before it.
__global__ __launch_bounds__(kThreads) void kv4_keep_kernel(tbn_kv4_pool p, tbn_kv_index ix, const int32_t *__restrict__ base, const int32_t *__restrict__ picks,
                                                            int width, const int32_t *__restrict__ counts) {
    __shared__ uint32_t keys[kBlock][kMaxDim / 8], exps[2][kBlock][2];
    __shared__ uint8_t values[kBlock][kMaxDim];
    __shared__ int32_t from[kBlock];
    const int tid = threadIdx.x, s = blockIdx.y, head = blockIdx.x, shift = __ffs(p.page) - 1, D = p.dim, NF = D / 16, EW = D <= 128 ? 1 : 2;
    const int failed = *ix.status, len = len_in(ix.lens[s], int64_t(ix.max_pages) << shift), b = base[s];
    const int n = b < 0 || b > len ? 0 : min(min(counts[s], width), len - b);
    if (failed || n <= 0) return;
    const int32_t *row = ix.table + int64_t(s) * ix.max_pages;
    // where key `at` of the sequence lies among the layer's keys
    auto place_of = [&](int at) {
        return (int64_t(page_in(row[at >> shift], static_cast<int>(p.n_pages))) * p.kv_heads + head) * p.page + (at & (p.page - 1));
    };
    uint32_t *kc = static_cast<uint32_t *>(p.k), *vc = static_cast<uint32_t *>(p.v), *ke = reinterpret_cast<uint32_t *>(p.k_exp), *ve = reinterpret_cast<uint32_t *>(p.v_exp);
    for (int j0 = 0; j0 < n; j0 += kBlock) {
        const int m = min(kBlock, n - j0), t0 = b + j0;
        __syncthreads();
        if (tid < m) {
            const int pick = picks[int64_t(s) * width + j0 + tid];
            from[tid] = pick > j0 + tid && pick < len - b ? b + pick : -1;   // -1: stays where it is, or is not there
        }
        __syncthreads();
        for (int i = tid; i < m * (D / 8); i += kThreads) {
            const int r = i / (D / 8), c = i - r * (D / 8);
            if (from[r] >= 0) keys[r][c] = kc[place_of(from[r]) * (D / 8) + c];
        }
        for (int i = tid; i < 2 * m * EW; i += kThreads) {
            const int which = i / (m * EW), r = i / EW % m, c = i % EW;
            if (from[r] >= 0) exps[which][r][c] = (which ? ve : ke)[place_of(from[r]) * EW + c];
        }
        for (int i = tid; i < m * D; i += kThreads) {
            const int r = i / D, d = i - r * D, f = from[r];
            if (f < 0) continue;
            const int64_t at = place_of(f);
            const int in = static_cast<int>(at & (kBlock - 1));
            values[r][d] = (vc[(at - in) * (D / 8) + kv4_value_word(in >> 3, d, NF)] >> (4 * (in & 7))) & 15u;
        }
        __syncthreads();
        for (int i = tid; i < m * (D / 8); i += kThreads) {
            const int r = i / (D / 8), c = i - r * (D / 8);
            if (from[r] >= 0) kc[place_of(t0 + r) * (D / 8) + c] = keys[r][c];
        }
        for (int i = tid; i < 2 * m * EW; i += kThreads) {
            const int which = i / (m * EW), r = i / EW % m, c = i % EW;
            if (from[r] >= 0) (which ? ve : ke)[place_of(t0 + r) * EW + c] = exps[which][r][c];
        }
        const int o0 = t0 >> 3, octets = ((t0 + m + 7) >> 3) - o0;
        for (int i = tid; i < octets * D; i += kThreads) {   // a word of eight keys: those of this round are put in
            const int o = i / D, d = i - o * D, at = (o0 + o) * 8;
            uint32_t mine = 0, w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = at + e - t0;
                if (r < 0 || r >= m || from[r] < 0) continue;
                mine |= 15u << (4 * e);
                w |= static_cast<uint32_t>(values[r][d]) << (4 * e);
            }
            if (!mine) continue;
            const int64_t place = place_of(at);
            const int in = static_cast<int>(place & (kBlock - 1));
            uint32_t *to = vc + (place - in) * (D / 8) + kv4_value_word(in >> 3, d, NF);
            *to = (*to & ~mine) | w;
        }
    }
}

// blocks that n keys can touch: one more than they fill
unsigned blocks_of(int32_t n) { return static_cast<unsigned>((int64_t(n) + kBlock - 2) / kBlock + 1); }

template <typename T>
void launch_append_typed(const tbn_kv4_pool &p, const tbn_kv_index &ix, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *cu,
                         int total, int32_t most, hipStream_t stream) {
    kv4_by_groups(p.dim, [&](auto nb) {
        hipLaunchKernelGGL((kv4_append_kernel<T, nb()>), dim3(blocks_of(most), p.kv_heads, ix.n_seqs), dim3(kWave), 0, stream, p, ix, static_cast<const T *>(k), k_stride,
                           static_cast<const T *>(v), v_stride, cu, total);
    });
}

template <typename T>
void launch_read_typed(const tbn_kv4_pool &p, const tbn_kv_index &ix, void *k, void *v, const int32_t *cu, int total, int32_t most, hipStream_t stream) {
    kv4_by_groups(p.dim, [&](auto nb) {
        hipLaunchKernelGGL((kv4_read_kernel<T, nb()>), dim3(blocks_of(most), p.kv_heads, ix.n_seqs), dim3(kWave), 0, stream, p, ix, static_cast<T *>(k), static_cast<T *>(v), cu,
                           total);
    });
}

}  // namespace

tbn_status launch_kv4_append(const tbn_kv4_pool &p, const tbn_kv_index &ix, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                             tbn_dtype dt, const int32_t *cu_new, int64_t total, int32_t max_new, hipStream_t stream) {
    if (dt == TBN_F32) launch_append_typed<float>(p, ix, k_new, k_stride, v_new, v_stride, cu_new, static_cast<int>(total), max_new, stream);
    else launch_append_typed<uint16_t>(p, ix, k_new, k_stride, v_new, v_stride, cu_new, static_cast<int>(total), max_new, stream);
    return check_launch("tbn_kv4_append");
}

tbn_status launch_kv4_read(const tbn_kv4_pool &p, const tbn_kv_index &ix, void *k, void *v, tbn_dtype dt, const int32_t *cu, int64_t total, int32_t most,
                           hipStream_t stream) {
    if (dt == TBN_F32) launch_read_typed<float>(p, ix, k, v, cu, static_cast<int>(total), most, stream);
    else launch_read_typed<uint16_t>(p, ix, k, v, cu, static_cast<int>(total), most, stream);
    return check_launch("tbn_kv4_read");
}

tbn_status launch_kv4_copy_pages(const tbn_kv4_pool &p, const int32_t *src, const int32_t *dst, int64_t n, const int32_t *count, hipStream_t stream) {
    const int codes = p.kv_heads * p.page * (p.dim / 2), exps = p.kv_heads * p.page * exponent_bytes(p.dim);   // at most 2^24
    const int64_t items = n * 2 * ((codes + kPiece - 1) / kPiece + (exps + kPiece - 1) / kPiece);
    hipLaunchKernelGGL(kv4_copy_kernel, dim3(static_cast<unsigned>(items < 8192 ? items : 8192)), dim3(256), 0, stream, p, src, dst, n, count, codes, exps);
    return check_launch("tbn_kv4_copy_pages");
}

tbn_status launch_kv4_keep(const tbn_kv4_pool &p, const tbn_kv_index &ix, const int32_t *base, const int32_t *picks, int32_t width, const int32_t *counts,
                           hipStream_t stream) {
    hipLaunchKernelGGL(kv4_keep_kernel, dim3(p.kv_heads, ix.n_seqs), dim3(kThreads), 0, stream, p, ix, base, picks, width, counts);
    return check_launch("tbn_kv4_keep");
}

}  // namespace tbn
