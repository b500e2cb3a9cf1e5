"""Every address from which the attention kernels load keys and values lies in the head of a listed page, on the CPU: the statements that form
the addresses are cut from the kernels' sources and run on the host for every instance, width, page size, lane and step, with the loads replaced
by a check of the 16 bytes that they would read (and of where in LDS they would write)."""
import os
import re
import subprocess

import pytest

from paper_2407_12075_amd import build as hip_build

_COMMON = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>
using std::min;
using std::max;
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_readfirstlane(x) (x)
constexpr int kWave = 64, kAttnWaves = 4, kAttnThreads = 256;
struct u32x4_t { uint32_t x, y, z, w; };
struct int2 { int x, y; };
static int __ffs(int v) { return __builtin_ffs(v); }
struct Pool { const void *k, *v; int64_t n_pages; int kv_heads, dim, page; };
struct Args { Pool p; };
static std::vector<char> k_bytes, v_bytes;
static std::vector<int> in_list;      // pages that the sequence holds
static int64_t head_bytes, heads, the_head;
static const uint32_t kZeros[4] = {0, 0, 0, 0}, kNothing[4] = {0, 0, 0, 0};
static long reads, faults;
static char what[64];
static void fault(const char *why, int64_t at) {
    if (faults++ < 5) std::printf("%s: %s at byte %lld\n", what, why, (long long)at);
}
// 16 bytes of keys (of values) that a load reads
static void touch(const void *from, bool keys) {
    ++reads;
    const char *at = static_cast<const char *>(from);
    if (keys && (from == static_cast<const void *>(kZeros) || from == static_cast<const void *>(kNothing))) return;
    const std::vector<char> &b = keys ? k_bytes : v_bytes;
    const int64_t o = at - b.data();
    if (o < 0 || o + 16 > int64_t(b.size())) return fault(keys ? "keys outside the pool" : "values outside the pool", o);
    const int64_t head = o / head_bytes, page = head / heads;
    if (head % heads != the_head || o % head_bytes + 16 > head_bytes || std::find(in_list.begin(), in_list.end(), int(page)) == in_list.end())
        fault(keys ? "keys of another head or page" : "values of another head or page", o);
}
static Args make(int D, int P, int KV, int n_pages, int elem, std::vector<int> pages) {
    head_bytes = int64_t(D) * P * elem;
    heads = KV;
    the_head = KV - 1;
    k_bytes.assign(head_bytes * KV * n_pages, 0);
    v_bytes.assign(head_bytes * KV * n_pages, 0);
    in_list = pages;
    return Args{{k_bytes.data(), v_bytes.data(), n_pages, KV, D, P}};
}
"""


def cut(text, begin, end):
    assert text.count(begin) == 1, f"{text.count(begin)} places read {begin!r}"
    at = text.index(begin)
    return text[at:text.index(end, at)]


def source(name):
    with open(os.path.join(hip_build.CSRC, name)) as f:
        return f.read()


def run(tmp_path, program):
    src, exe = tmp_path / "addresses.cpp", tmp_path / "addresses"
    src.write_text(_COMMON + program)
    subprocess.run(["g++", "-O1", "-std=c++17", "-w", str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert done.returncode in (0, 1), done.stdout
    return done.returncode == 0, done.stdout


_ROWS = r"""
typedef uint16_t *lds_at;
static uint16_t *lds_k, *lds_v;
static int64_t lds_k_size, lds_v_size;
static void arrive(const void *from, void *to) {
    uint16_t *t = static_cast<uint16_t *>(to);
    const bool keys = t >= lds_k && t < lds_k + lds_k_size;
    if (keys ? t + kWave * 8 > lds_k + lds_k_size : t < lds_v || t + kWave * 8 > lds_v + lds_v_size) fault("outside of LDS", 0);
    touch(from, keys);
}
#define __builtin_amdgcn_global_load_lds(from, to, bytes, offset, aux) arrive(from, to)
@KEY_OF_ROW@
template <int DP, int RW, bool EVEN>
static void instance(int D, int P, int keys) {
    @CONSTANTS@
    const int n_entries = (keys + P - 1) / P;
    std::vector<int> listed;
    for (int i = 0; i < n_entries; ++i) listed.push_back(n_entries - i);   // the first of them is the pool's last page
    std::snprintf(what, sizeof what, "<%d, %d, %d> D %d P %d keys %d", DP, RW, EVEN, D, P, keys);
    const Args a = make(D, P, 3, n_entries + 1, 2, listed);
    std::vector<uint16_t> tiles(KEYS * PITCH + DP * KEYS);
    lds_k = tiles.data();
    lds_k_size = KEYS * PITCH;
    lds_v = lds_k + lds_k_size;
    lds_v_size = DP * KEYS;
    for (int tid = 0; tid < kAttnThreads; ++tid) {
        const int lane = tid & 63, wave = tid >> 6, shift = __ffs(P) - 1, entries = n_entries, KV = a.p.kv_heads;
        const struct { int head; } blk = {KV - 1};
        @STAGING@
        for (int i = 0; i < (keys + KEYS - 1) / KEYS; ++i) request(i, lds_k, lds_v);
    }
}
template <int DP>
static void width(int from) {
    for (int D = from; D <= DP; D += 8)
        for (int P : {32, 64, 128})
            for (int keys : {1, 33, 64, 100, 128, 129, 256, 257}) {
                if (D == DP) instance<DP, 2, true>(D, P, keys), instance<DP, 4, true>(D, P, keys);
                else instance<DP, 2, false>(D, P, keys), instance<DP, 4, false>(D, P, keys);
            }
}
int main() {
    width<64>(8);
    width<96>(72);
    width<128>(104);
    width<256>(136);
    std::printf("%ld reads, %ld faults\n", reads, faults);
    return faults != 0;
}
"""


def rows_program():
    text = source("tbn_kv_rows.hip")
    constants = cut(text, "    constexpr int KW = kAttnWaves / RW", "    // two buffers of each")
    staging = cut(text, "    // where this lane's pieces come from", "    f32x16_t o[ND];")
    key = cut(text, "__device__ __forceinline__ int key_of_row(int r)", "\n")
    staging = re.sub(r"__attribute__\(\(address_space\(\d\)\)\) ", "", staging)
    return _ROWS.replace("@KEY_OF_ROW@", key).replace("@CONSTANTS@", constants).replace("@STAGING@", staging)


def test_staged_kernel_reads_what_the_pages_hold(tmp_path):
    """The launch takes the narrowest of 64, 96, 128 and 256 channels that holds the head, its even form where they are equal."""
    dispatch = re.findall(r"a\.p\.dim <= (\d+)\) launch_dim<(\d+)>", source("tbn_kv_rows.hip"))
    assert dispatch == [("64", "64"), ("96", "96"), ("128", "128")]
    good, out = run(tmp_path, rows_program())
    assert good, out


def test_the_check_sees_a_row_that_is_padded_in_lds(tmp_path):
    """96 channels lie 128 apart in LDS: pieces 12 to 15 of a row are not the head's, though the head has every channel of the instance."""
    program = rows_program()
    assert program.count("FULL || ") == 1 and program.count("if (!FULL)") == 1
    good, out = run(tmp_path, program.replace("FULL || ", "EVEN || ").replace("if (!FULL)", "if (!EVEN)"))
    assert not good and "<96, 2, 1> D 96" in out and "keys outside the pool" in out


_PICKED = r"""
static uint32_t t0_at, t1_at, box_bytes;
static bool sends_keys;
static void landed(uint32_t to) {
    const bool in0 = to >= t0_at && to + kWave * 16 <= t0_at + box_bytes, in1 = to >= t1_at && to + kWave * 16 <= t1_at + box_bytes;
    if (!in0 && !in1) fault("outside of LDS", to);
}
static void send(uint32_t to, const void *base, uint32_t lane_offset) { landed(to), touch(static_cast<const char *>(base) + lane_offset, sends_keys); }
static void send(uint32_t to, const void *from) { landed(to), touch(from, sends_keys); }
@KEY_OF_ROW@
template <int DP, bool EVEN, bool PAIRS>
static void instance(int D, int P, int n_entries) {
    @CONSTANTS@
    std::vector<int2> listed;
    std::vector<int> pages;
    for (int i = 0; i < n_entries; ++i) listed.push_back(int2{2 * i, 1}), pages.push_back(n_entries - i);
    std::snprintf(what, sizeof what, "<%d, %d, %d> D %d P %d entries %d", DP, EVEN, PAIRS, D, P, n_entries);
    const Args a = make(D, P, 3, n_entries + 1, 2, pages);
    box_bytes = BUF * 2;
    for (int tid = 0; tid < kAttnThreads; ++tid) {
        const int lane = tid & 63, wave = tid >> 6, shift = __ffs(P) - 1, entries = n_entries, KV = a.p.kv_heads;
        const struct { int head; } blk = {KV - 1};
        static uint16_t b0[kAttnWaves][BUF], b1[kAttnWaves][BUF];
        @STAGING@
        t0_at = to0;
        t1_at = to1;
        for (int i = wave; i < units; i += kAttnWaves) {
            Unit u = {{kp, kp}, {vp, vp}, {0, 0}, {0, 0}};
            unit_of(i, u);
            for (int t = 0; t < 2; ++t) {
                sends_keys = true;
                request_k(t ? to1 : to0, u.k[t]);
                sends_keys = false;
                request_v(t ? to1 : to0, u, t);
            }
        }
    }
}
template <int DP>
static void width(int from) {
    for (int D = from; D <= DP; D += 8)
        for (int entries : {1, 2, 3, 9}) {
            if (D == DP) instance<DP, true, true>(D, 32, entries), instance<DP, true, false>(D, 64, entries), instance<DP, true, false>(D, 128, entries);
            else instance<DP, false, true>(D, 32, entries), instance<DP, false, false>(D, 64, entries), instance<DP, false, false>(D, 128, entries);
        }
}
int main() {
    width<64>(8);
    width<128>(72);
    width<256>(136);
    std::printf("%ld reads, %ld faults\n", reads, faults);
    return faults != 0;
}
"""


def test_kernel_of_shared_picks_reads_what_the_pages_hold(tmp_path):
    text = source("tbn_kv_picked.hip")
    constants = cut(text, "    constexpr int BUF = 32 * DP;", "    __shared__")
    staging = cut(text, "    struct Unit {", "    f32x16_t o[ND];")
    staging = re.sub(r"__attribute__\(\(address_space\(\d\)\)\) ", "", staging)
    key = cut(text, "__device__ __forceinline__ int key_of_row(int r)", "\n")
    good, out = run(tmp_path, _PICKED.replace("@KEY_OF_ROW@", key).replace("@CONSTANTS@", constants).replace("@STAGING@", staging))
    assert good, out


_DIRECT = r"""
static bool loads_keys;
static u32x4_t read16(const void *at) { touch(at, loads_keys); return u32x4_t{}; }
template <typename T> struct Elem;
template <> struct Elem<uint16_t> { static constexpr int kStep = 32, kOf = 8, kTiles = 2; };
template <> struct Elem<float> { static constexpr int kStep = 16, kOf = 4, kTiles = 1; };
template <typename T, int DP, bool EVEN>
static void instance(int D, int P) {
    using E = Elem<T>;
    constexpr int KS = E::kStep, OF = E::kOf, NF = DP / 16;
    std::snprintf(what, sizeof what, "<%d bytes, %d, %d> D %d P %d", int(sizeof(T)), DP, EVEN, D, P);
    const Args a = make(D, P, 3, 3, sizeof(T), {0, 2});
    for (int lane = 0; lane < 64; ++lane) {
        const int n = lane & 15, g = lane >> 4, shift = __ffs(P) - 1, KV = a.p.kv_heads, head = KV - 1, entries = 1;
        @LOADS@
        u32x4_t k[NF];
        for (int page : in_list)
            for (int off = 0; off < P; off += KS) {
                loads_keys = true;
                load_k(k, page, off);
                loads_keys = false;
                load_v(k, page, off);
            }
    }
}
template <typename T, int DP>
static void width(int from) {
    for (int D = from; D <= DP; D += 8)
        for (int P : {32, 64, 128}) {
            if (D == DP) instance<T, DP, true>(D, P);
            else instance<T, DP, false>(D, P);
        }
}
int main() {
    width<float, 64>(8), width<float, 128>(72), width<float, 256>(136);
    width<uint16_t, 64>(8), width<uint16_t, 128>(72), width<uint16_t, 256>(136);
    std::printf("%ld reads, %ld faults\n", reads, faults);
    return faults != 0;
}
"""


def test_kernel_of_few_rows_reads_what_the_pages_hold(tmp_path):
    loads = cut(source("tbn_kv_attention.hip"), "    const int64_t page_elems = int64_t(P) * D;", "    // step i of this stretch")
    loads, n = re.subn(r"\*reinterpret_cast<const u32x4_t \*>\(", "read16(", loads)
    assert n == 2
    good, out = run(tmp_path, _DIRECT.replace("@LOADS@", loads))
    assert good, out
