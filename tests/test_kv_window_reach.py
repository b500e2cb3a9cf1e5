"""The keys that a workgroup goes through in a call with a window never are more than its plan has stretches for, on the CPU: the functions that say
where its pages end and how many keys are planned are cut from the kernels' header and run on the host, with sequences that have more tokens than the call's
max_q among them (their parts would lie behind the workspace)."""
from tests.test_kv_addresses import cut, run, source

_PROGRAM = r"""
struct WindowArgs { int32_t sink, size; };
struct KvQueries { int32_t max_q, heads; int64_t max_len; };
struct tbn_kv_pool { int kv_heads, page; };
struct AttentionArgs { tbn_kv_pool p; const uint32_t *mask; WindowArgs window; };
@SPAN@
@KEYS_END@
@WITHIN@
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
@WINDOW_KEYS@
int main() {
    const uint32_t some = 0;
    for (int G : {1, 3, 8, 40})
        for (int P : {32, 64, 128})
            for (int sink : {0, 1, 4, 33, 64, 300, 1 << 30})
                for (int size : {1, 2, 31, 64, 65, 500, 1 << 30})
                    for (int max_q : {1, 2, 7, 33, 200})
                        for (int tokens : {1, 2, 6, 33, 34, 100, 201, 700})
                            for (int before : {0, 1, 31, 63, 64, 500, 1000, 3000})
                                for (int masked : {0, 1})
                                    for (int cut_off : {0, 40}) {
                                        if (masked && max_q > size) continue;
                                        const int T = min(tokens, max_q), R = T * G, most = 4096;
                                        const int len = min(before + tokens, most - cut_off);   // keys beyond max_len are not read
                                        AttentionArgs a{{2, P}, masked ? &some : nullptr, {sink, size}};
                                        KvQueries q{max_q, 2 * G, most - cut_off};
                                        const Span v{0, T, len, max(len - tokens, 0)};
                                        const int64_t planned = window_keys(a.p, q, sink, size, masked);
                                        for (int tile : {16, 32, 64, 128})
                                            for (int base = 0; base < R; base += tile) {
                                                const Within w = within_of(a, v, base, min(base + tile, R) - 1, G, __ffs(P) - 1);
                                                ++reads;
                                                std::snprintf(what, sizeof what, "G%d P%d sink%d size%d q%d/%d len%d m%d", G, P, sink, size, tokens, max_q, len, masked);
                                                if (w.end > planned) fault("more keys than planned", w.end - planned);
                                                if (w.end > 0 && (w.key(w.end - 1) < 0 || w.key(w.end - 1) >= max(len, 1))) fault("a key that is not there", w.key(w.end - 1));
                                            }
                                    }
    std::printf("%ld tiles, %ld faults\n", reads, faults);
    return faults ? 1 : 0;
}
"""


def program():
    text = source("tbn_kv_attention.h")
    parts = {"SPAN": cut(text, "struct Span {", "__device__ __forceinline__ Span span_of"),
             "KEYS_END": cut(text, "__device__ __forceinline__ int keys_end(", "// The keys that the rows"),
             "WITHIN": cut(text, "struct Within {", "// The least key of a row's window"),
             "WINDOW_KEYS": cut(text, "inline int64_t window_keys(", "inline size_t workspace_of(")}
    out = _PROGRAM
    for name, part in parts.items():
        out = out.replace(f"@{name}@", part)
    return out


def test_no_more_keys_than_planned(tmp_path):
    fine, text = run(tmp_path, program())
    assert fine and "tiles, 0 faults" in text, text
    assert int(text.split()[0]) > 100000


def test_the_check_sees_a_plan_that_is_too_short(tmp_path):
    fine, text = run(tmp_path, program().replace("+ 2 * p.page)", "- 2 * p.page)"))
    assert not fine and "more keys than planned" in text
