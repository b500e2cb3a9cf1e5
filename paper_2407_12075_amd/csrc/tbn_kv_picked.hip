// Attention over picked blocks for many queries at a time (prompt chunks; bfloat16).  Mathematics and
// parts as in tbn_kv_attention.hip.
//
// Queries one by one read every page they pick for themselves.  That traffic comes from L2 and is bound by the L1: operands loaded
// straight into registers put neighbouring lanes on different rows, 9.6 TB/s over the GPU, against 30 TB/s for whole lines.  So
//   - 32 rows, that is 32 / G neighbouring queries, share a workgroup, which goes through the union of their picks; a page's
//     keys enter a row's sums only if its query picked the page;
//   - keys and values come in whole lines into LDS and from there into registers (piece index xor row, as in tbn_kv_rows.hip).
//
// The four waves of a workgroup take units of 64 keys (of one page, or two pages of 32) in turn and do not wait for each other: each has two buffers of its own, which
// hold in turn the two halves of a unit's keys (32 keys each) and the two halves of its values (half of the channels each).  A
// buffer's next contents are requested as soon as it has been read: S of one half of the keys, the other half, softmax, both halves
// of the channels.  The waves' sums meet in LDS at the end.
//
// A row whose query did not pick the unit has weights of 0.  Times an infinite value or not a number that would be no number, so if
// a sum ends up as one the workgroup does its work again, more slowly, with such values counted apart.
#include "tbn_kv_attention.h"

namespace tbn {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kUnions = 1024;   // picks of a workgroup's queries together, at most

__device__ __attribute__((aligned(16))) const uint32_t kNothing[4] = {0, 0, 0, 0};   // channels beyond the head's

__device__ __forceinline__ f32x16_t mma(u32x4_t a, u32x4_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// key of row r of a tile of 32 (tbn_kv_rows.hip)
__device__ __forceinline__ int key_of_row(int r) { return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3); }

// One piece of each lane from memory to LDS, 64 in a row from `to` on (an LDS address), past the registers.  Written out so that the
// compiler does not put waits of its own in front of reads of the other buffer; each use is followed by the kernel's own waits, oldest
// requests first.  (A cycle lies between writing m0 and its use.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is always clobbered
__device__ __forceinline__ void send(uint32_t to, const void *base, uint32_t lane_offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(lane_offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void send(uint32_t to, const void *from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// DP: channels (dim <= DP; EVEN: equal).  PAIRS: pages of 32 keys.  a.row_tiles tiles of `queries` queries.
template <int DP, bool EVEN, bool PAIRS>
__global__ __launch_bounds__(kAttnThreads, DP == 256 ? 1 : 2) void kv_picked_kernel(AttentionArgs a, int queries) {
    constexpr int BUF = 32 * DP;                 // elements: 32 keys of DP channels, or DP / 2 channels of 64 keys
    constexpr int KP = DP / 8, NP = BUF / 8 / kWave;   // pieces of a row of K; pieces of a lane
    constexpr int NQ = DP / 16, ND = DP / 32;
    __shared__ __attribute__((aligned(16))) uint16_t b0[kAttnWaves][BUF], b1[kAttnWaves][BUF];
    __shared__ int2 listed[kUnions];             // block and the queries that picked it
    __shared__ int pages[kUnions];
    __shared__ float4 totals[kAttnWaves][32];
    __shared__ int counts[kAttnWaves];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int s = blockIdx.y, H = a.q.heads, KV = a.p.kv_heads, G = H / KV, D = EVEN ? DP : a.p.dim, P = PAIRS ? 32 : a.p.page, shift = __ffs(P) - 1;
    const Span v = span_of(a, s);
    const Block blk = block_of(a);
    const int t_first = blk.row_tile * queries;
    if (t_first >= v.T) return;
    const int T = min(queries, v.T - t_first), R = T * G;    // this workgroup's queries and rows
    const int32_t *table = a.ix.table + int64_t(s) * a.ix.max_pages;

    // the union of the picks: a word per block in the buffers' place (at most b0's words: picked_queries)
    uint32_t *member = reinterpret_cast<uint32_t *>(&b0[0][0]);
    const int last = min(v.len, v.prefix + t_first + T) - 1, blocks = last < 0 ? 0 : (last >> shift) + 1;
    for (int i = tid; i < blocks; i += kAttnThreads) member[i] = 0;
    __syncthreads();
    for (int i = tid; i < T * a.n_select; i += kAttnThreads) {
        const int t = i / a.n_select, own = min(v.len - 1, v.prefix + t_first + t);
        const int b = a.picks[(int64_t(v.t0 + t_first + t) * KV + blk.head) * a.n_select + (i - t * a.n_select)];
        if (b >= 0 && (b << shift) <= own && b < blocks) atomicOr(&member[b], 1u << t);
    }
    __syncthreads();
    int entries = 0;
    for (int i0 = 0; i0 < blocks; i0 += kAttnThreads) {
        const uint32_t who = i0 + tid < blocks ? member[i0 + tid] : 0u;
        const uint64_t some = __ballot(who != 0);
        if (lane == 0) counts[wave] = __popcll(some);
        __syncthreads();
        int at = entries + __popcll(some & ((uint64_t(1) << lane) - 1));
#pragma unroll
        for (int u = 0; u < kAttnWaves; ++u) {
            at += u < wave ? counts[u] : 0;
            entries += counts[u];
        }
        if (who) {
            listed[at] = make_int2(i0 + tid, static_cast<int>(who));
            pages[at] = page_in(table[i0 + tid], static_cast<int>(a.p.n_pages));
        }
        __syncthreads();
    }

    const int in = min(n, R - 1), mine = in / G, end = min(v.len, v.prefix + t_first + mine + 1);   // this lane's row: its query, where its keys end
    const int64_t at = int64_t(v.t0 + t_first + mine) * H + blk.head * G + (in - mine * G);
    u32x4_t q[NQ];
    {
        const uint16_t *src = static_cast<const uint16_t *>(a.q.q) + (v.t0 + t_first + mine) * a.q.q_stride + (blk.head * G + in - mine * G) * D;
#pragma unroll
        for (int f = 0; f < NQ; ++f) q[f] = *reinterpret_cast<const Elem<uint16_t>::u32x4_any *>(src + (EVEN ? f * 16 + 8 * h : min(f * 16 + 8 * h, D - 8)));
#pragma unroll
        for (int f = 0; f < NQ; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[f][e] = n < R && (EVEN || f * 16 + 8 * h < D) ? q[f][e] ^ a.flip : 0u;
    }

    struct Unit {   // its halves of 32 keys: where keys and values are, the first key, who picked it
        const uint16_t *k[2], *v[2];
        int key[2];
        uint32_t who[2];
    };
    const int64_t page_elems = int64_t(P) * D;
    const uint16_t *kp = static_cast<const uint16_t *>(a.p.k) + blk.head * page_elems, *vp = static_cast<const uint16_t *>(a.p.v) + blk.head * page_elems;
    // Piece j of this lane in a buffer of keys is row U + lane / KP, U = 64 j / KP, and there piece (lane % KP) xor (row & 7).  Both parts of
    // the row have bits of their own, so the key of the row is the sum of theirs and the piece c0 xor (U & 7): what differs between
    // pieces is the same for all lanes, but for the few values of U & 7.
    const int c0 = (lane % KP) ^ ((lane / KP) & 7);
    const int v_piece = (lane % 8) ^ (lane / 8);   // of a channel's 64 keys; PAIRS: the first four are the first page's
    const uint32_t k_lane = key_of_row(lane / KP) * D * 2, v_lane = ((lane / 8) * P + (PAIRS ? v_piece & 3 : v_piece) * 8) * 2;
    auto request_k = [&](uint32_t to, const uint16_t *k) {   // 32 keys from k on
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            constexpr int kStep = kWave / KP;
            const int c = c0 ^ ((j * kStep) & 7);
            const uint16_t *row = k + key_of_row(j * kStep) * D;
            if (EVEN) send(to + j * (kWave * 16), row, k_lane + c * 16);
            else send(to + j * (kWave * 16), c * 8 < D ? reinterpret_cast<const char *>(row) + (k_lane + c * 16) : reinterpret_cast<const char *>(kNothing));
        }
    };
    auto request_v = [&](uint32_t to, const Unit &u, int half) {   // channels DP / 2 * half on of its 64 keys
        const char *mine = PAIRS ? reinterpret_cast<const char *>(v_piece < 4 ? u.v[0] : u.v[1]) + v_lane : nullptr;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int d = half * (DP / 2) + 8 * j;   // channels beyond the head's: any, their sums are dropped
            const int at = (EVEN ? d : min(d, D - 8)) * P;
            if (PAIRS) send(to + j * (kWave * 16), mine + at * 2);
            else send(to + j * (kWave * 16), u.v[0] + at, v_lane);
        }
    };

    uint16_t *const w0 = b0[wave], *const w1 = b1[wave];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    const uint32_t to0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)w0)), to1 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)w1));
    const int units = PAIRS ? (entries + 1) >> 1 : entries << (shift - 6);
    auto unit_of = [&](int i, Unit &u) {
#pragma unroll
        for (int t = 0; t < (PAIRS ? 2 : 1); ++t) {
            const int entry = PAIRS ? 2 * i + t : i >> (shift - 6), off = PAIRS ? 0 : (i & ((1 << (shift - 6)) - 1)) * 64;
            const int use = PAIRS ? min(entry, entries - 1) : entry;   // behind the last page: it again, picked by nobody
            const int2 e = listed[use];
            const int block = __builtin_amdgcn_readfirstlane(e.x);
            const int64_t page = int64_t(__builtin_amdgcn_readfirstlane(pages[use])) * (page_elems * KV);
            u.who[t] = use == entry ? static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(e.y)) : 0u;
            u.k[t] = kp + page + off * D;
            u.v[t] = vp + page + off;
            u.key[t] = (block << shift) + off;
        }
        if (!PAIRS) {
            u.who[1] = u.who[0];
            u.k[1] = u.k[0] + 32 * D;
            u.v[1] = u.v[0];
            u.key[1] = u.key[0] + 32;
        }
    };

    f32x16_t o[ND];
    float m, l, z;
    for (int careful = 0; careful < 2; ++careful) {
#pragma unroll
        for (int f = 0; f < ND; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[f][e] = 0.f;
        m = -INFINITY;
        l = z = 0.f;
        __syncthreads();   // the list is complete, the buffers are free
        Unit now = {{kp, kp}, {vp, vp}, {0, 0}, {0, 0}};
        int i = wave;
        if (i < units) {
            unit_of(i, now);
            request_k(to0, now.k[0]);
            request_k(to1, now.k[1]);
        }
        for (; i < units; i += kAttnWaves) {
            Unit next = now;
            if (i + kAttnWaves < units) unit_of(i + kAttnWaves, next);   // (behind the last one: this one again)
            f32x16_t p[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint16_t *buf = t ? w1 : w0;
#pragma unroll
                for (int e = 0; e < 16; ++e) p[t][e] = 0.f;
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NP) : "memory");   // this buffer's pieces are older than the other's
                u32x4_t x[NQ];
#pragma unroll
                for (int f = 0; f < NQ; ++f) x[f] = *reinterpret_cast<const u32x4_t *>(buf + n * DP + ((2 * f + h) ^ (n & 7)) * 8);
#pragma unroll
                for (int f = 0; f < NQ; ++f) p[t] = mma(x[f], q[f], p[t]);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the buffer has been read
                request_v(t ? to1 : to0, now, t);
            }
            const bool member[2] = {static_cast<bool>((now.who[0] >> mine) & 1u), static_cast<bool>((now.who[1] >> mine) & 1u)};
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (__any(now.key[t] + 32 > end)) {   // some row's keys end in this half
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint32_t bits = first_bits(end - (now.key[t] + 16 * u + 8 * h));
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[t][8 * u + e] = (bits >> e) & 1u ? p[t][8 * u + e] : -INFINITY;
                    }
                }
                float most = p[t][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) most = fmaxf(most, p[t][e]);
                top = member[t] ? fmaxf(top, most) : top;
            }
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
            u32x4_t pw[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t only = member[t] ? ~0u : 0u;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = exp2_of(fmaf(p[t][8 * u + 2 * e], a.c, -from)), y = exp2_of(fmaf(p[t][8 * u + 2 * e + 1], a.c, -from));
                        sum += x + y;
                        pw[2 * t + u][e] = two_bf16(x, y) & only;
                        z = add_two_bf16(pw[2 * t + u][e], z);
                    }
                l += member[t] ? sum : 0.f;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint16_t *buf = t ? w1 : w0;
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NP) : "memory");
                if (careful) {
#pragma unroll 1
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t seen = (u < 2 ? member[0] : member[1]) ? first_bits(end - ((u < 2 ? now.key[0] : now.key[1]) + 16 * (u & 1) + 8 * h)) : 0u;
                        const u32x4_t ones = Elem<uint16_t>::ones(seen);
#pragma unroll
                        for (int f = 0; f < ND / 2; ++f) {
                            const int d = f * 32 + n;
                            u32x4_t *piece = reinterpret_cast<u32x4_t *>(buf + d * 64 + ((2 * u + h) ^ (d & 7)) * 8), finite, kinds;
                            Elem<uint16_t>::part(*piece, finite, kinds);
                            *piece = finite;   // this wave's buffer, and each piece is one lane's
                            f32x16_t found;
#pragma unroll
                            for (int e = 0; e < 16; ++e) found[e] = 0.f;
                            found = mma(kinds, ones, found);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[t * (ND / 2) + f][e] += limit_of(found[e]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                u32x4_t x[ND / 2 * 4];
#pragma unroll
                for (int f = 0; f < ND / 2; ++f)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int d = f * 32 + n;
                        x[f * 4 + u] = *reinterpret_cast<const u32x4_t *>(buf + d * 64 + ((2 * u + h) ^ (d & 7)) * 8);
                    }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int f = 0; f < ND / 2; ++f) o[t * (ND / 2) + f] = mma(x[f * 4 + u], pw[u], o[t * (ND / 2) + f]);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                request_k(t ? to1 : to0, next.k[t]);
            }
            now = next;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way into the buffers any more
        if (careful) break;
        bool odd = false;
        if (n < R)
#pragma unroll
            for (int f = 0; f < ND; ++f)
#pragma unroll
                for (int e = 0; e < 16; ++e) odd |= !(fabsf(o[f][e]) < INFINITY);
        if (!__syncthreads_or(odd)) break;
    }

    {   // the other half of each row's keys lies in the lane 32 away
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(z), __float_as_uint(z), false, false);
        l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        z = __uint_as_float(u[0]) + __uint_as_float(u[1]);
    }
    // The waves' sums: half of the channels at a time, four boxes of 32 rows; wave w adds up the rows' channels 4 (..) + its share.
    if (h == 0) totals[wave][n] = make_float4(m, l, z, 0.f);
    __syncthreads();
    float best = totals[0][n].x;
#pragma unroll
    for (int u = 1; u < kAttnWaves; ++u) best = fmaxf(best, totals[u][n].x);
    const float mine_f = m == best ? 1.f : exp2_of(m - best);
    l = z = 0.f;
#pragma unroll
    for (int u = 0; u < kAttnWaves; ++u) {
        const float4 t = totals[u][n];
        const float f = t.x == best ? 1.f : exp2_of(t.x - best);
        l += t.y * f;
        z += t.z * f;
    }
    constexpr int kBox = ND / 2 * 4;   // pieces of four channels of a lane and half
    f32x4_t *box = reinterpret_cast<f32x4_t *>(b0[wave]);
    static_assert(kBox * kWave * 16 <= BUF * 2, "a buffer holds half of a wave's sums");
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        __syncthreads();   // the boxes may still be read
#pragma unroll
        for (int f = 0; f < ND / 2; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x16_t &x = o[t * (ND / 2) + f];
                box[(f * 4 + i) * kWave + lane] = f32x4_t{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]} * mine_f;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kBox / kAttnWaves; ++j) {
            const int c = j * kAttnWaves + wave, d = t * (DP / 2) + (c >> 2) * 32 + 8 * (c & 3) + 4 * h;
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < kAttnWaves; ++u) sum += reinterpret_cast<const f32x4_t *>(b0[u])[c * kWave + lane];
            if (n < R && (EVEN || d < D)) store_sums<uint16_t>(a, 0, at, d, sum, best, l, z);
        }
    }
}

template <int DP, bool PAIRS>
void launch_page(const AttentionArgs &a, int queries, dim3 grid, hipStream_t stream) {
    if (a.p.dim == DP) hipLaunchKernelGGL((kv_picked_kernel<DP, true, PAIRS>), grid, dim3(kAttnThreads), 0, stream, a, queries);
    else hipLaunchKernelGGL((kv_picked_kernel<DP, false, PAIRS>), grid, dim3(kAttnThreads), 0, stream, a, queries);
}

template <int DP>
void launch_dim(const AttentionArgs &a, int queries, dim3 grid, hipStream_t stream) {
    if (a.p.page == 32) launch_page<DP, true>(a, queries, grid, stream);
    else launch_page<DP, false>(a, queries, grid, stream);
}

}  // namespace

// Queries that share a workgroup, 0 where queries go one by one: float32, heads or picks of which 32 rows or the
// list hold fewer than two queries, tables longer than the buffers have words, or so few workgroups that the GPU is all but empty.
int picked_queries(const tbn_kv_pool &p, const tbn_kv_index &ix, const KvQueries &q, int32_t n_select) {
    if (p.dt != TBN_BF16) return 0;
    const int G = q.heads / p.kv_heads, words = p.dim <= 64 ? 4096 : p.dim <= 128 ? 8192 : 16384;
    int queries = G <= 32 ? 32 / G : 0;
    if (queries > kUnions / n_select) queries = kUnions / n_select;
    if (queries > q.max_q) queries = q.max_q;
    if (queries < 2 || ix.max_pages > words) return 0;
    // fewer queries together while that leaves CUs idle (the union of 64 queries' picks, eight by eight, is 46 us of one workgroup's work)
    auto groups = [&] { return (q.total_q + queries - 1) / queries * p.kv_heads; };
    while (queries > 3 && groups() < 256) queries /= 2;
    return groups() >= 64 ? queries : 0;
}

void launch_kv_picked(const AttentionArgs &a, int queries, dim3 grid, hipStream_t stream) {
    if (a.p.dim <= 64) launch_dim<64>(a, queries, grid, stream);
    else if (a.p.dim <= 128) launch_dim<128>(a, queries, grid, stream);
    else launch_dim<256>(a, queries, grid, stream);
}

}  // namespace tbn
