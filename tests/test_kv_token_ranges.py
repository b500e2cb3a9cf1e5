"""The tokens that a sequence of a call has lie within the call's, whatever the array of first tokens holds, on the CPU: the function that every kernel takes them from is cut from the header
and run with the ends of 32 bits, whose plain differences wrap around to ranges far behind the arrays."""
import os
import re

from paper_2407_12075_amd import build as hip_build
from tests.test_kv_addresses import cut, run, source

_PROGRAM = r"""
@TOKENS_IN@
int main() {
    const int32_t ends[] = {INT32_MIN, INT32_MIN + 1, -100000, -2, -1, 0, 1, 2, 63, 64, 1000, 1 << 30, INT32_MAX - 3, INT32_MAX - 1, INT32_MAX};
    for (int64_t total : {int64_t(0), int64_t(1), int64_t(64), int64_t(999), int64_t(1) << 30})
        for (int32_t a : ends)
            for (int32_t b : ends) {
                const int32_t cu[3] = {-7, a, b};
                int32_t first;
                const int64_t n = tokens_in(cu, 1, total, first);
                ++reads;
                if (first < 0 || (n > 0 && first + n > total)) fault("tokens that the call does not have", n);
                if (a >= 0 && b >= a && b <= total && (first != a || n != b - a)) fault("not the tokens of the sequence", n);
            }
    std::printf("%ld ranges, %ld faults\n", reads, faults);
    return faults ? 1 : 0;
}
"""


def test_ranges(tmp_path):
    program = _PROGRAM.replace("@TOKENS_IN@", cut(source("tbn_kv.h"), "__device__ __forceinline__ int32_t tokens_in(", "__device__ __forceinline__ int32_t len_in("))
    fine, text = run(tmp_path, program)
    assert fine and "1125 ranges, 0 faults" in text, text


def test_every_kernel_takes_them_from_there():
    """No other place reads where a sequence ends; where one begins, only the search for a token's sequence and reads of a sequence that is known to have tokens."""
    for name in sorted(os.listdir(hip_build.CSRC)):
        if name.startswith(("tbn_kv", "tbn_verify")) and name.endswith((".hip", ".h")):
            text = source(name)
            ends = re.findall(r"\bcu(?:_q|_new)?\[s \+ 1\]", text)
            assert len(ends) == (1 if name == "tbn_kv.h" else 0), (name, ends)
