"""Every address from which the attention kernels load the cache in 4 bits lies in the head of a listed page, on the CPU: the statements that form the
addresses are cut from the kernels' sources and run on the host for every width, page size, lane and step, with the loads replaced by a check."""
import re

from tests.test_kv_addresses import cut, run, source

_COMMON = r"""
template <int N> struct Words { uint32_t w[N]; };
struct Pool4 { const void *k, *v; const int8_t *summary; const float *step; int64_t n_pages; int kv_heads, dim, page; };
struct Args4 { Pool4 p; };
static std::vector<char> arrays[4];   // codes of keys and values, exponents of both
static int64_t head_size[2];          // bytes of a head of a page: codes, exponents
template <int N> Words<N> words_at(const void *from) {
    ++reads;
    const char *at = static_cast<const char *>(from);
    for (int i = 0; i < 4; ++i) {
        const int64_t o = at - arrays[i].data(), size = head_size[i / 2];
        if (o < 0 || o >= int64_t(arrays[i].size())) continue;
        const int64_t head = o / size, page = head / heads;
        if (o % 4 || head % heads != the_head || o % size + 4 * N > size || std::find(in_list.begin(), in_list.end(), int(page)) == in_list.end())
            fault("another head or page", o);
        return Words<N>{};
    }
    fault("outside of the pool", 0);
    return Words<N>{};
}
static Args4 make4(int D, int P, int KV, int n_pages, std::vector<int> pages) {
    head_size[0] = int64_t(D) * P / 2;
    head_size[1] = int64_t(P) * (D <= 128 ? 4 : 8);
    for (int i = 0; i < 4; ++i) arrays[i].assign(head_size[i / 2] * KV * n_pages, 0);
    heads = KV;
    the_head = KV - 1;
    in_list = pages;
    return Args4{{arrays[0].data(), arrays[1].data(), reinterpret_cast<int8_t *>(arrays[2].data()), reinterpret_cast<float *>(arrays[3].data()), n_pages, KV, D, P}};
}
"""

_FEW = r"""
template <int NB> static void instance(int P) {
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2;
    std::snprintf(what, sizeof what, "<%d> P %d", NB, P);
    const Args4 a = make4(D, P, 3, 4, {0, 3});
    for (int lane = 0; lane < 64; ++lane) {
        const int n = lane & 15, g = lane >> 4, KV = a.p.kv_heads, head = KV - 1;
        @LOADS@
        Step x;
        for (int page : in_list)
            for (int off = 0; off < P; off += 32) load_k(x, page, off), load_v(x, page, off);
    }
}
"""

_ROWS = r"""
template <int NB> static void instance(int P) {
    constexpr int D = 32 * NB, NF = 2 * NB, EW = NB <= 4 ? 1 : 2, KEYS = 64;
    for (int keys : {1, 31, 33, 64, 65, 100, 128, 257}) {
        std::snprintf(what, sizeof what, "<%d> P %d keys %d", NB, P, keys);
        const int entries = (keys + P - 1) / P, shift = __ffs(P) - 1;
        std::vector<int> listed;
        for (int i = 0; i < entries; ++i) listed.push_back(entries - i);
        const Args4 a = make4(D, P, 3, entries + 1, listed);
        for (int tid = 0; tid < kAttnThreads; ++tid) {
            const int KV = a.p.kv_heads;
            const struct { int head; } blk = {KV - 1};
            @LOADS@
            Step x;
            for (int i = 0; i < (keys + KEYS - 1) / KEYS; ++i) load(x, i);
        }
    }
}
"""

_MAIN = r"""
template <int NB> static void pages() { for (int P : {32, 64, 128}) instance<NB>(P); }
int main() {
    pages<1>(), pages<2>(), pages<3>(), pages<4>(), pages<5>(), pages<6>(), pages<7>(), pages<8>();
    std::printf("%ld reads, %ld faults\n", reads, faults);
    return faults != 0 || reads == 0;
}
"""


def program(body, name, begin, end):
    loads, n = re.subn(r"\*reinterpret_cast<const Words<(\w+)> \*>\(", r"words_at<\1>(", cut(source(name), begin, end))
    assert n == 4
    return _COMMON + body.replace("@LOADS@", loads) + _MAIN


def few():
    return program(_FEW, "tbn_kv4_attention.hip", "    struct Step {", "    const int sub_shift")


def rows():
    return program(_ROWS, "tbn_kv4_rows.hip", "    const int part = tid >> 7", "    auto store = ")


def test_kernel_of_few_rows_reads_what_the_pages_hold(tmp_path):
    good, out = run(tmp_path, few())
    assert good, out


def test_staged_kernel_reads_what_the_pages_hold(tmp_path):
    good, out = run(tmp_path, rows())
    assert good, out


def test_the_check_sees_a_step_too_far(tmp_path):
    text = few()
    assert text.count("off + k_key") == 1
    good, out = run(tmp_path, text.replace("off + k_key", "off + k_key + 1"))
    assert not good and "another head or page" in out
    text = rows()
    assert text.count("min(off >> shift, entries - 1)") == 1 and text.count("8 * kg + e") == 1
    good, out = run(tmp_path, text.replace("8 * kg + e", "8 * kg + e + 1"))
    assert not good
