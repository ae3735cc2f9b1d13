"""Outputs of the verification that lie over its inputs are refused before anything touches a GPU.  The addresses are made up."""
import ctypes as C

import pytest

from paper_2407_20143_b200 import _lib as L
from paper_2407_20143_b200 import api

AT = 1 << 20
N, DRAFTS = 3, 4  # sequences, drafts of each
PLACES = {"drafts": 8 * N * DRAFTS, "uniform": 4 * N * (DRAFTS + 1), "temperature": 4 * N, "tokens": 8 * N * (DRAFTS + 1), "accepted": 4 * N}


def verify(**at):
    a = {**{name: AT + 4096 * (i + 1) for i, name in enumerate(PLACES)}, **at}
    rows = L.VocabRowsC(AT + (1 << 16), 1000, 100, 2, 0)
    return L.lib().bcp_verify_drafts(C.addressof(rows), C.addressof(rows), N, DRAFTS, 100, a["drafts"], a["uniform"], a["temperature"], 0, a["tokens"], a["accepted"], None)


@pytest.mark.parametrize("output,over", [(o, i) for o in ("tokens", "accepted") for i in ("drafts", "uniform", "temperature")] + [("tokens", "accepted")])
def test_overlap_is_refused(output, over):
    first = AT + (1 << 18)
    for shift in (0, 4, PLACES[over] - 4, 4 - PLACES[output]):
        assert verify(**{over: first, output: first + shift}) == api.ERR_DST_ALIAS
        assert b"overlap" in L.lib().bcp_last_error()


def test_drafts_inside_the_tokens_of_one_sequence():
    # out[:, :n] as the drafts of a call that writes out: contiguous for a single sequence
    rows = L.VocabRowsC(AT + (1 << 16), 0, 100, 2, 0)
    for at in (AT, AT + 8):
        assert L.lib().bcp_verify_drafts(C.addressof(rows), None, 1, 4, 100, at, AT + 4096, None, 0, AT, AT + 8192, None) == api.ERR_DST_ALIAS
