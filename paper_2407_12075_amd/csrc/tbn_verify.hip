// Verification of drafted tokens: which of them the target accepts, and the token that follows.
//
// At an accepted token x (the first of a sequence to begin with) r = target[x], m = 1.  The tokens that hang on x are asked in order: c is accepted where
// u_c m q(c) < r(c), q = draft[x] (without a draft q is 1 at c and 0 elsewhere); if it is not, r = max(r - m q, 0), m = sum of r, and the next one is
// asked.  When none is left the token that follows is the first whose prefix sum of r is above u sum(r).
//
// Everything is in binary64: a product of a few 24-bit numbers is exact or off by 2^-53, so that a border is hit only by numbers that lie on it, and
// sums of a row are off by about 1e-16 of it, whatever their order.  (It is fixed all the same.)  No product is fused with a sum: r has one value.
//
// The path needs two numbers of each drafted token, loaded side by side; it is walked by every wave alike, in LDS.  A sum over a row is needed where a
// token was refused and another one hangs on the same (with a draft), and at the end.  What bounds it is the latency of a handful of dependent
// loads and, for many sequences with large vocabularies, the bytes of the last rows: there slices of a row are summed by many workgroups, each of which
// walks the path for itself, and a second launch finds the slice and the token in it.
//
// What is left of a row is made from the target's again wherever it is needed, by the refusals in their order.  Those of many siblings would be applied again for
// each of them, so every kKept refusals the sum of the row leaves it in the workspace, in binary64 (the same numbers, therefore), and the next ones go on from there:
// a refusal costs one pass over the row, however many there were before.
#include <algorithm>

#include "tbn_kv.h"

namespace tbn {

namespace {

// Without the draft's probabilities; with them; with them where sequences have tokens enough for rows to be kept.  (Instances of their own: where no row can be kept
// the branches would cost 16 trees of 10 tokens on 50000 elements 3 us of 29.)
enum Draft { kNoDraft, kDraft, kKeeping };

constexpr int kBig = 1024, kSmall = 256;   // threads of a workgroup
constexpr int kSlice = 4096;
constexpr int kDraw = kSlice / 16;         // threads of the last launch's workgroups

struct VerifyArgs {
    const float *target, *draft;
    int64_t target_stride, draft_stride;
    const int32_t *tokens, *parents;
    const float *u;
    const int32_t *cu;
    int32_t *picks, *counts, *next;
    int64_t total;
    int32_t max_q, n_seqs, vocab;
    // split rows: sums of slices, where each sequence's path ends and what was refused there
    double *parts;
    int2 *ends;       // row of the target (-1: no tokens), refused ones
    double *refused;  // (sequence, max_q): m with a draft, else the token
    int32_t slices;
    double *left;     // rows that kKept refusals and more have left (left_row)
};

// Refusals at one token after which what is left is kept: 2047 siblings on 131072 elements take 226 ms (130 with 32), but trees of up to 65 tokens keep the faster
// instances (4 trees of 48 tokens on 32000 elements: 28.4 us, 30.4 with 32).  A row that is kept belongs to a sequence of kKept + 2 tokens at least, so the rows are
// few: an eight-byte number for 66 of the target's at most.
constexpr int kKept = 64, kKeepers = kKept + 2;

// The row of a sequence that begins at token t0 and has kKeepers tokens or more: no two of them have the same.
__device__ __forceinline__ double *left_row(const VerifyArgs &a, int t0) { return a.left + int64_t(t0 / kKeepers) * a.vocab; }

// What is left of a row of the target: of p, or of `left`, which is what earlier refusals have made of it, after n more.
struct Rest {
    const float *p, *q;
    const double *refused;
    int n;
    const double *left;
};

__device__ __forceinline__ double count(float p) { return p > 0.f ? static_cast<double>(p) : 0.; }   // negative numbers and not-a-numbers are 0

// r of element v after one refusal.
template <Draft DRAFT>
__device__ __forceinline__ double refuse(double r, double q, double refused, int v) {
#pragma clang fp contract(off)
    if constexpr (DRAFT != kNoDraft) {
        const double part = refused * q, d = r - part;
        return d > 0. ? d : 0.;
    } else {
        return refused == static_cast<double>(v) ? 0. : r;
    }
}

// r of one element, whose p and q are at hand
template <Draft DRAFT>
__device__ __forceinline__ double left_of(const Rest &x, int v, float p, float q) {
    double r = DRAFT == kKeeping && x.left ? x.left[v] : count(p);
    for (int i = 0; i < x.n; ++i) r = refuse<DRAFT>(r, count(q), x.refused[i], v);
    return r;
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void four_at(const float *row, int v, int hi, float (&f)[4]) {
    if (v + 4 <= hi) {
        const f32x4_any w = *reinterpret_cast<const f32x4_any *>(row + v);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = v + e < hi ? row[v + e] : 0.f;
    }
}

// r of J times four elements, from v + j * step on, those below hi (others 0).
template <Draft DRAFT, int J>
__device__ __forceinline__ void fours_of(const Rest &x, int v, int step, int hi, double (&r)[J][4]) {
    float p[J][4], q[J][4];
    auto take_off = [&] {
        for (int i = 0; i < x.n; ++i) {
            const double refused = x.refused[i];
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) r[j][e] = refuse<DRAFT>(r[j][e], DRAFT ? count(q[j][e]) : 0., refused, v + j * step + e);
        }
    };
    if (DRAFT == kKeeping && x.left) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            four_at(x.q, v + j * step, hi, q[j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[j][e] = v + j * step + e < hi ? x.left[v + j * step + e] : 0.;
        }
        return take_off();
    }
#pragma unroll
    for (int j = 0; j < J; ++j) four_at(x.p, v + j * step, hi, p[j]);
    if (DRAFT && x.n) {
#pragma unroll
        for (int j = 0; j < J; ++j) four_at(x.q, v + j * step, hi, q[j]);
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[j][e] = count(p[j][e]);
    take_off();
}

__device__ __forceinline__ double sum_of_wave(double s) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d);
    return s;
}

// Sum of a wave's elements [lo, hi).  KEEP: they go to `keep` where that is not null (it may be x.left: a thread writes what it has read).
template <Draft DRAFT, bool KEEP>
__device__ __forceinline__ double sum_of(const Rest &x, int lo, int hi, double *keep) {
    constexpr int kVectors = 4;
    double s = 0.;
    for (int base = lo; base < hi; base += kVectors * 4 * kWave) {
        const int own = base + 4 * (threadIdx.x & 63);
        double r[kVectors][4];
        fours_of<DRAFT, kVectors>(x, own, 4 * kWave, hi, r);
        if (KEEP && keep) {
#pragma unroll
            for (int j = 0; j < kVectors; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = own + j * 4 * kWave + e;
                    if (at < hi) keep[at] = r[j][e];
                }
        }
#pragma unroll
        for (int j = 0; j < kVectors; ++j) s += (r[j][0] + r[j][1]) + (r[j][2] + r[j][3]);
    }
    return sum_of_wave(s);
}

struct DrawLds {
    double sums[kBig / kWave];
    int token, last;
};

__device__ __forceinline__ bool drawable(double sum) { return sum > 0. && sum < INFINITY; }

// Every wave of the workgroup takes an equal run of [lo, hi); their sums in order.  Every thread calls it.
template <Draft DRAFT, int THREADS, bool KEEP = false>
__device__ __forceinline__ double sums_of_waves(const Rest &x, int lo, int hi, DrawLds &l, int &run, double *keep = nullptr) {
    constexpr int kWaves = THREADS / kWave;
    const int wave = threadIdx.x >> 6;
    run = ((hi - lo + kWaves - 1) / kWaves + 3) & ~3;
    const int from = min(lo + wave * run, hi), to = min(from + run, hi);
    __syncthreads();   // the sums may still be read from the call before
    const double s = sum_of<DRAFT, KEEP>(x, from, to, keep);
    if ((threadIdx.x & 63) == 0) l.sums[wave] = s;
    __syncthreads();
    double all = 0.;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += l.sums[w];
    return all;
}

// Narrows [lo, hi) to the run in which the prefix sum passes `at`, which becomes what is left of it there: the first run whose end is above, else
// the last one that holds anything.
template <int N>
__device__ __forceinline__ void narrow(const double *sums, int run, int &lo, int &hi, double &at) {
    double before = 0., start = 0.;
    int pick = -1, last = -1;
    double last_start = 0.;
    for (int w = 0; w < N; ++w) {
        const double s = sums[w];
        if (pick < 0 && s > 0.) {
            last = w;
            last_start = before;
            if (before + s > at) {
                pick = w;
                start = before;
            }
        }
        before += s;
    }
    if (pick < 0) {
        pick = max(last, 0);
        start = last_start;
    }
    at -= start;
    lo = min(lo + pick * run, hi);
    hi = min(lo + run, hi);
}

__device__ __forceinline__ double prefix_of_wave(double s) {   // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const double below = __shfl_up(s, d);
        if (lane >= d) s += below;
    }
    return s;
}

// The first element of [lo, hi) whose prefix sum is above `at`, else the last one that is not 0 (-1: none).  SHARE: `at` is a share of the sum, and the
// result -2 where that is no positive finite number.  At most kEach elements of each thread, which are loaded once; every thread calls it.
constexpr int kEach = 16;
template <Draft DRAFT, bool SHARE, int THREADS>
__device__ int find_in(const Rest &x, int lo, int hi, double at, DrawLds &l) {
    constexpr int kWaves = THREADS / kWave;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, from = lo + tid * kEach;
    double r[kEach / 4][4], own = 0.;
    fours_of<DRAFT, kEach / 4>(x, from, 4, hi, r);
#pragma unroll
    for (int i = 0; i < kEach / 4; ++i) own += (r[i][0] + r[i][1]) + (r[i][2] + r[i][3]);
    const double incl = prefix_of_wave(own);
    __syncthreads();   // the sums may still be read from the call before
    if (lane == 63) l.sums[wave] = incl;
    if (tid == 0) {
        l.token = INT32_MAX;
        l.last = -1;
    }
    __syncthreads();
    double before = 0., sum = 0.;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before = w == wave ? sum : before;
        sum += l.sums[w];
    }
    if (SHARE) {
        if (!drawable(sum)) return -2;   // the same for all
        at *= sum;
    }
    double s = before + (incl - own);
    int mine = INT32_MAX, last = -1;
#pragma unroll
    for (int i = 0; i < kEach / 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s += r[i][e];
            if (r[i][e] > 0.) {
                last = from + 4 * i + e;
                if (s > at) mine = min(mine, last);
            }
        }
    const uint64_t hit = __ballot(mine != INT32_MAX), any = __ballot(last >= 0);
    if (hit && lane == __ffsll(static_cast<unsigned long long>(hit)) - 1) atomicMin(&l.token, mine);
    if (any && lane == 63 - __clzll(static_cast<long long>(any))) atomicMax(&l.last, last);
    __syncthreads();
    return l.token != INT32_MAX ? l.token : l.last;
}

// The token of [lo, hi) at the share u of its sum; -2 where that is no positive finite number.
template <Draft DRAFT, int THREADS>
__device__ int draw_in(const Rest &x, int lo, int hi, double u, DrawLds &l) {
    if (hi - lo <= THREADS * kEach) return find_in<DRAFT, true, THREADS>(x, lo, hi, u, l);
    int run;
    double sum = sums_of_waves<DRAFT, THREADS>(x, lo, hi, l, run);
    if (!drawable(sum)) return -2;
    double at = u * sum;
    narrow<THREADS / kWave>(l.sums, run, lo, hi, at);
    while (hi - lo > THREADS * kEach) {
        (void)sums_of_waves<DRAFT, THREADS>(x, lo, hi, l, run);
        narrow<THREADS / kWave>(l.sums, run, lo, hi, at);
    }
    return find_in<DRAFT, false, THREADS>(x, lo, hi, at, l);
}

// What the walk leaves behind.
struct End {
    int at, n;   // place of the last accepted token, tokens refused there
    int count;   // accepted ones
};
// What was refused at the token of place `at` lies from place at + 1 on: those tokens' own places are above it and below the next accepted one's, so
// the list of one token never overwrites another's, which a slower wave may still read.

struct Nodes {   // of a sequence, in LDS
    double *refused;
    float *p, *q, *u;
    int32_t *parent, *token;
};

__device__ __forceinline__ Nodes nodes_at(void *lds, int most) {
    Nodes n;
    n.refused = static_cast<double *>(lds);
    n.p = reinterpret_cast<float *>(n.refused + most);
    n.q = n.p + most;
    n.u = n.q + most;
    n.parent = reinterpret_cast<int32_t *>(n.u + most);
    n.token = n.parent + most;
    return n;
}
constexpr int kNodeBytes = 28;
constexpr int kMaxNodes = 2048;

// Every wave walks alike.  PASSES: a row is summed where a token was refused and another one hangs on the same.
template <Draft DRAFT, bool PASSES, int THREADS>
__device__ End walk(const VerifyArgs &a, int t0, int T, const Nodes &nodes, DrawLds &l, int32_t *picks) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int j = tid; j < T; j += THREADS) {
        const int parent = j == 0 ? -1 : a.parents ? a.parents[t0 + j] : j - 1, token = a.tokens[t0 + j];
        const bool in = token >= 0 && token < a.vocab && parent >= 0 && parent < j;
        const float p = in ? a.target[(t0 + parent) * a.target_stride + token] : 0.f;
        nodes.q[j] = !DRAFT ? 1.f : in ? a.draft[(t0 + parent) * a.draft_stride + token] : 0.f;
        nodes.p[j] = p;
        nodes.u[j] = a.u[t0 + j];
        nodes.parent[j] = parent;
        nodes.token[j] = token;
    }
    __syncthreads();
    End end{0, 0, 1};
    if (picks && tid == 0) picks[0] = 0;
    double m = 1.;
    bool known = true;   // m is the sum of what is left
    int kept = 0;        // refusals at end.at that the row in the workspace holds
    auto refusals = [&](const float *p, const float *q) {
        return Rest{p, q, nodes.refused + end.at + 1 + kept, end.n - kept, kept ? left_row(a, t0) : nullptr};
    };
    for (int after = 0;;) {
        int c = -1;   // the next one that hangs on it
        for (int j0 = (after + 1) & ~63; j0 < T; j0 += kWave) {
            const int j = j0 + lane;
            const uint64_t here = __ballot(j < T && j > after && nodes.parent[min(j, T - 1)] == end.at);
            if (here) {
                c = j0 + __ffsll(static_cast<unsigned long long>(here)) - 1;
                break;
            }
        }
        if (c < 0) break;
        after = c;
        if (PASSES && !known) {
            const Rest x = refusals(a.target + (t0 + end.at) * a.target_stride, a.draft + (t0 + end.at) * a.draft_stride);
            const bool keep = DRAFT == kKeeping && end.n % kKept == 0;   // of at least kKeepers tokens: this one, kKept that were refused, and c
            int run;
            m = sums_of_waves<DRAFT, THREADS, DRAFT == kKeeping>(x, 0, a.vocab, l, run, keep ? left_row(a, t0) : nullptr);
            known = true;
            if (keep) kept = end.n;
        }
        Rest one = refusals(nullptr, nullptr);
        if (DRAFT == kKeeping && (nodes.token[c] < 0 || nodes.token[c] >= a.vocab)) one.left = nullptr;   // such tokens have p = q = 0
        const double r = left_of<DRAFT>(one, nodes.token[c], nodes.p[c], nodes.q[c]);
        const double q = nodes.q[c] > 0.f ? static_cast<double>(nodes.q[c]) : 0.;
        const double limit = DRAFT ? m * q : m;
        if (static_cast<double>(nodes.u[c]) * limit < r) {
            if (picks && tid == 0) picks[end.count] = c;
            end = End{c, 0, end.count + 1};
            m = 1.;
            known = true;
            kept = 0;
        } else {
            nodes.refused[end.at + 1 + end.n++] = DRAFT ? m : static_cast<double>(nodes.token[c]);   // every wave writes the same
            if (DRAFT) known = false;
            else m = m - r > 0. ? m - r : 0.;
        }
    }
    if (picks)
        for (int j = end.count + tid; j < a.max_q; j += THREADS) picks[j] = -1;
    return end;
}

// What is left at the end of a walk, of which `refused` holds all refusals.  The row was summed after each of them but the last.
template <Draft DRAFT>
__device__ __forceinline__ Rest rest_of(const VerifyArgs &a, int t0, int row, const double *refused, int n) {
    const int kept = DRAFT == kKeeping && n > kKept ? (n - 1) / kKept * kKept : 0;
    return Rest{a.target + row * a.target_stride, DRAFT ? a.draft + row * a.draft_stride : nullptr, refused + kept, n - kept, kept ? left_row(a, t0) : nullptr};
}
// the target's row itself
__device__ __forceinline__ Rest whole_row(const Rest &x) { return Rest{x.p, x.q, nullptr, 0, nullptr}; }

__device__ __forceinline__ bool sequence_at(const VerifyArgs &a, int s, int &t0, int &T) {
    T = min(tokens_in(a.cu, s, a.total, t0), a.max_q);
    return T > 0;
}

__device__ __forceinline__ void nothing(const VerifyArgs &a, int s) {
    for (int j = threadIdx.x; j < a.max_q; j += blockDim.x) a.picks[int64_t(s) * a.max_q + j] = -1;
    if (threadIdx.x == 0) {
        a.counts[s] = 0;
        a.next[s] = -1;
    }
}

// A workgroup for each sequence does everything.
template <Draft DRAFT, int THREADS>
__global__ __launch_bounds__(THREADS) void verify_kernel(VerifyArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ DrawLds l;
    const int s = blockIdx.x;
    int t0, T;
    if (!sequence_at(a, s, t0, T)) return nothing(a, s);
    const Nodes nodes = nodes_at(lds, a.max_q);
    const End end = walk<DRAFT, DRAFT != kNoDraft, THREADS>(a, t0, T, nodes, l, a.picks + int64_t(s) * a.max_q);
    const Rest x = rest_of<DRAFT>(a, t0, t0 + end.at, nodes.refused + end.at + 1, end.n);
    const double u = static_cast<double>(nodes.u[0]);
    int token = draw_in<DRAFT, THREADS>(x, 0, a.vocab, u, l);
    if (token == -2) token = max(draw_in<DRAFT, THREADS>(whole_row(x), 0, a.vocab, u, l), -1);   // nothing is left
    if (threadIdx.x == 0) {
        a.counts[s] = end.count;
        a.next[s] = token;
    }
}

// Rows in slices.  First launch: each workgroup walks the path (WALK; else verify_walk_kernel has) and sums its slice of the last row.
template <Draft DRAFT, bool WALK>
__global__ __launch_bounds__(kSmall) void verify_slices_kernel(VerifyArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ DrawLds l;
    const int s = blockIdx.y, slice = blockIdx.x, tid = threadIdx.x;
    Rest x;
    if constexpr (WALK) {
        int t0, T;
        if (!sequence_at(a, s, t0, T)) {
            if (slice == 0) {
                nothing(a, s);
                if (tid == 0) a.ends[s] = make_int2(-1, 0);
            }
            return;
        }
        const Nodes nodes = nodes_at(lds, a.max_q);
        const End end = walk<DRAFT, false, kSmall>(a, t0, T, nodes, l, slice == 0 ? a.picks + int64_t(s) * a.max_q : nullptr);
        if (slice == 0) {
            for (int i = tid; i < end.n; i += kSmall) a.refused[int64_t(s) * a.max_q + i] = nodes.refused[end.at + 1 + i];
            if (tid == 0) {
                a.counts[s] = end.count;
                a.ends[s] = make_int2(t0 + end.at, end.n);
            }
        }
        x = rest_of<DRAFT>(a, t0, t0 + end.at, nodes.refused + end.at + 1, end.n);
    } else {
        const int2 end = a.ends[s];
        if (end.x < 0) return;
        x = rest_of<DRAFT>(a, max(a.cu[s], 0), end.x, a.refused + int64_t(s) * a.max_q, end.y);
    }
    const int lo = slice * kSlice, hi = min(lo + kSlice, a.vocab);
    int run;
    const double sum = sums_of_waves<DRAFT, kSmall>(x, lo, hi, l, run);
    if (tid == 0) a.parts[int64_t(s) * a.slices + slice] = sum;
}

template <Draft DRAFT>
__global__ __launch_bounds__(kBig) void verify_walk_kernel(VerifyArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ DrawLds l;
    const int s = blockIdx.x;
    int t0, T;
    if (!sequence_at(a, s, t0, T)) {
        nothing(a, s);
        if (threadIdx.x == 0) a.ends[s] = make_int2(-1, 0);
        return;
    }
    const Nodes nodes = nodes_at(lds, a.max_q);
    const End end = walk<DRAFT, DRAFT != kNoDraft, kBig>(a, t0, T, nodes, l, a.picks + int64_t(s) * a.max_q);
    for (int i = threadIdx.x; i < end.n; i += kBig) a.refused[int64_t(s) * a.max_q + i] = nodes.refused[end.at + 1 + i];
    if (threadIdx.x == 0) {
        a.counts[s] = end.count;
        a.ends[s] = make_int2(t0 + end.at, end.n);
    }
}

// Last launch: the slice and the token in it.
template <Draft DRAFT>
__global__ __launch_bounds__(kDraw) void verify_draw_kernel(VerifyArgs a) {
    __shared__ DrawLds l;
    const int s = blockIdx.x, lane = threadIdx.x & 63;
    const int2 end = a.ends[s];
    if (end.x < 0) return;
    const int t0 = max(a.cu[s], 0);
    const Rest x = rest_of<DRAFT>(a, t0, end.x, a.refused + int64_t(s) * a.max_q, end.y);
    const double *parts = a.parts + int64_t(s) * a.slices;
    double sum = 0.;
    for (int i = lane; i < a.slices; i += kWave) sum += parts[i];
    sum = sum_of_wave(sum);
    const double u = static_cast<double>(a.u[t0]);
    int token = -1;
    if (drawable(sum)) {
        double at = u * sum;
        // the first slice whose end is above, else the last one that holds anything; every wave alike
        int pick = -1, last = 0;
        double before = 0., last_start = 0.;
        for (int base = 0; base < a.slices && pick < 0; base += kWave) {
            const double own = base + lane < a.slices ? parts[base + lane] : 0.;
            double incl = own;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const double below = __shfl_up(incl, d);
                if (lane >= d) incl += below;
            }
            const uint64_t hit = __ballot(own > 0. && before + incl > at), any = __ballot(own > 0.);
            if (any) {
                const int from = hit ? __ffsll(static_cast<unsigned long long>(hit)) - 1 : 63 - __clzll(static_cast<long long>(any));
                last = base + from;
                last_start = before + __shfl(incl - own, from);
                if (hit) pick = last;
            }
            before += __shfl(incl, 63);
        }
        at -= last_start;
        const int lo = last * kSlice, hi = min(lo + kSlice, a.vocab);
        static_assert(kSlice <= kDraw * kEach, "a slice fits the registers of a workgroup");
        token = find_in<DRAFT, false, kDraw>(x, lo, hi, at, l);
    } else if (end.y) {   // nothing is left
        token = max(draw_in<DRAFT, kDraw>(whole_row(x), 0, a.vocab, u, l), -1);
    }
    if (threadIdx.x == 0) a.next[s] = token;
}

// Rows go in slices where they are long and the sequences are too few to give every CU one.
int slices_of(int64_t vocab, int64_t sequences) { return vocab > 16384 && sequences < 256 ? static_cast<int>((vocab + kSlice - 1) / kSlice) : 0; }

template <Draft DRAFT>
void launch(const VerifyArgs &a, hipStream_t stream) {
    const unsigned lds = static_cast<unsigned>(kNodeBytes * a.max_q);
    if (!a.slices) {
        // as few threads as hold the row in their registers: waiting for each other costs less (1024 elements: 7.2 us in place of 7.9)
        if (a.vocab <= kSmall * kEach) hipLaunchKernelGGL((verify_kernel<DRAFT, kSmall>), dim3(a.n_seqs), dim3(kSmall), lds, stream, a);
        else hipLaunchKernelGGL((verify_kernel<DRAFT, kBig>), dim3(a.n_seqs), dim3(kBig), lds, stream, a);
        return;
    }
    const dim3 grid(a.slices, a.n_seqs);
    if (DRAFT && a.parents) {   // rows may have to be summed on the way
        hipLaunchKernelGGL((verify_walk_kernel<DRAFT>), dim3(a.n_seqs), dim3(kBig), lds, stream, a);
        hipLaunchKernelGGL((verify_slices_kernel<DRAFT, false>), grid, dim3(kSmall), 0, stream, a);
    } else if constexpr (DRAFT != kKeeping) {
        hipLaunchKernelGGL((verify_slices_kernel<DRAFT, true>), grid, dim3(kSmall), lds, stream, a);
    }
    hipLaunchKernelGGL((verify_draw_kernel<DRAFT>), dim3(a.n_seqs), dim3(kDraw), 0, stream, a);
}

}  // namespace

int verify_most_tokens() { return kMaxNodes; }

// of the slices; of the rows that are kept behind them
static size_t slices_bytes(int64_t n_seqs, int64_t slices, int64_t max_q) { return slices ? 8 * static_cast<size_t>(n_seqs * (slices + 1 + max_q)) : 0; }
static size_t left_bytes(int64_t total, int64_t max_q, int64_t vocab) { return max_q >= kKeepers ? 8 * static_cast<size_t>(total / kKeepers * vocab) : 0; }

size_t verify_workspace(int64_t total, int32_t max_q, int32_t n_seqs, int64_t vocab) {
    return slices_bytes(n_seqs, slices_of(vocab, std::min<int64_t>(n_seqs, total)), max_q) + left_bytes(total, max_q, vocab);
}

tbn_status launch_verify(const VerifyCall &c, void *ws, hipStream_t stream) {
    VerifyArgs a{c.target, c.draft, c.target_stride, c.draft_stride, c.tokens, c.parents, c.u, c.cu_q, c.picks, c.counts, c.next, c.total, c.max_q, c.n_seqs,
                 static_cast<int32_t>(c.vocab), nullptr, nullptr, nullptr, slices_of(c.vocab, std::min<int64_t>(c.n_seqs, c.total)), nullptr};
    a.left = reinterpret_cast<double *>(static_cast<char *>(ws) + slices_bytes(a.n_seqs, a.slices, a.max_q));   // not looked at where there are none
    if (a.slices) {
        a.parts = static_cast<double *>(ws);
        a.refused = a.parts + int64_t(a.n_seqs) * a.slices;
        a.ends = reinterpret_cast<int2 *>(a.refused + int64_t(a.n_seqs) * a.max_q);
    }
    if (!a.draft) launch<kNoDraft>(a, stream);
    else if (!a.parents || !left_bytes(a.total, a.max_q, a.vocab)) launch<kDraft>(a, stream);
    else launch<kKeeping>(a, stream);
    return check_launch("tbn_verify");
}

}  // namespace tbn
