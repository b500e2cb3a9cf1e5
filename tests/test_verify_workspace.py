"""Bytes of the verification's workspace, on the CPU: rows that many refusals have left are kept for sequences that can have so many, and cost little beside
the target's rows."""
import pytest

from tests.test_kv_abi import FAKE, lib  # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("vocab", [1, 1000, 16384, 16385, 131072])
def test_rows_that_are_kept(lib, vocab):  # noqa: F811
    ask = lambda total, most, seqs: lib.tbn_verify_workspace_bytes(total, most, seqs, vocab)  # noqa: E731
    for total, most, seqs in ((26, 26, 1), (65, 65, 1), (640, 65, 40), (2000, 7, 300)):   # no sequence with more than 63 siblings
        assert ask(total, most, seqs) == ask(total, 1, seqs) + (8 * seqs * (most - 1) if ask(total, 1, seqs) else 0)
    for total, most, seqs in ((66, 66, 1), (2048, 2048, 1), (100000, 2048, 64), (5000, 100, 300)):
        more = ask(total, most, seqs) - ask(total, 65, seqs) - (8 * seqs * (most - 65) if ask(total, 1, seqs) else 0)
        assert more == 8 * vocab * (total // 66)
        assert more <= 4 * vocab * total / 30
    assert ask(60, 2048, 300) == ask(60, 65, 300) + (8 * 300 * (2048 - 65) if ask(60, 1, 300) else 0)   # fewer tokens than max_q says


def test_a_workspace_without_them_is_refused(lib):  # noqa: F811
    need = lib.tbn_verify_workspace_bytes(200, 200, 1, 1000)
    assert need == 3 * 8000
    call = lambda ws, n: lib.tbn_verify(FAKE, 1000, FAKE, 1000, FAKE, FAKE, FAKE, FAKE, 200, 200, 1, 1000, FAKE, FAKE, FAKE, ws, n, None)  # noqa: E731
    assert call(FAKE, need - 1) == 5 and call(None, need) == 5 and call(FAKE + 8, need) == 5
