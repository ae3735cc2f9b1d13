"""Host side of the operators of batches that share work: descriptors, refusals (all of them before anything touches a GPU), lists of axes.  The
addresses below are made up; every call must be refused before it could use one."""
import ctypes as C

import pytest

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import _lib as L
from paper_2407_20143_b200 import api

AT = 1 << 20  # a made-up address, aligned to everything
BF16, F16, F32, E4M3 = 2, 3, 1, 4
ref = lambda x: C.addressof(x) if x is not None else None  # noqa: E731


def heads(n=2, token_stride=128, head_stride=64, typ=BF16, data=AT):
    return L.HeadsC(data, token_stride, head_stride, n, typ)


def table(**k):
    a = dict(table=AT, n_positions=100, rot_dim=64, layout=0, status=None)
    return L.RopeTableC(*{**a, **k}.values())


def cache(**k):
    a = dict(k=AT, v=AT, k_scale=None, v_scale=None, page_stride=2048, head_stride=1024, token_stride=64, n_pages=4, page_size=16, n_heads=2,
             head_dim=64, format=BF16, reserved=0, status=None)
    return L.KvCacheC(*{**a, **k}.values())


OF_PAIR = (C.c_uint8 * 32)(*([0] * 16 + [1] * 16))
PAST = (C.c_uint8 * 32)(*([0] * 31 + [2]))


def axes(**k):
    a = dict(axis_of_pair=C.addressof(OF_PAIR), axis_stride=4, n_axes=2, reserved=0)
    return L.RopeAxesC(*{**a, **k}.values())


def code(rc):
    assert rc < 0 and L.lib().bcp_last_error()
    return rc


def test_descriptor_sizes():
    assert C.sizeof(L.RopeAxesC) == 24 and C.sizeof(L.VocabRowsC) == 32


@pytest.mark.parametrize("a", [None, axes(axis_of_pair=None), axes(n_axes=0), axes(n_axes=5), axes(reserved=1), axes(axis_stride=-1),
                               axes(axis_stride=(1 << 40) + 1), axes(n_axes=1), axes(axis_of_pair=C.addressof(PAST))])
def test_axes_refusals(a):
    h, t, c = heads(), table(), cache()
    assert code(L.lib().bcp_rope_axes(ref(h), ref(h), None, None, 64, 4, ref(t), ref(a), AT, 0, None)) == api.ERR_INVALID
    assert code(L.lib().bcp_kv_write_axes(ref(c), ref(h), ref(h), AT, 4, ref(t), ref(a), AT, None)) == api.ERR_INVALID
    assert code(L.lib().bcp_kv_write_axes(ref(c), ref(h), ref(h), AT, 4, None, ref(axes()), AT, None)) == api.ERR_INVALID


def test_what_calls_without_axes_refuse_is_refused_with_them():
    h, t, a = heads(), table(rot_dim=66), axes()
    assert code(L.lib().bcp_rope_axes(ref(h), ref(h), None, None, 64, 4, ref(t), ref(a), AT, 0, None)) == api.ERR_INVALID
    assert code(L.lib().bcp_rope_axes(ref(h), ref(h), None, None, 64, 4, ref(table()), ref(a), None, 0, None)) == api.ERR_INVALID


def test_lists_of_axes():
    assert bcp.rope_axes((2, 1, 3)) == [0, 0, 1, 2, 2, 2]
    assert bcp.rope_axes((2, 1, 3), interleaved=True) == [0, 1, 2, 0, 2, 2]
    assert bcp.rope_axes([4]) == [0, 0, 0, 0] == bcp.rope_axes([4], True)
    for bad in ((), (1, 0), (1, -1), (1, 1, 1, 1, 1)):
        with pytest.raises(bcp.BcpError):
            bcp.rope_axes(bad)


def shared(q=None, out=None, c=None, n=4, prefix_table=AT, prefix_stride=3, prefix_width=3, prefix_lengths=AT, starts=AT, prefixes=2, scale=1.0):
    q, out, c = q or heads(), out or heads(), c or cache()
    return code(L.lib().bcp_kv_attend_shared(ref(c), ref(q), ref(out), AT, n, prefix_table, prefix_stride, prefix_width, prefix_lengths, starts, prefixes, AT, 3, 3,
                                             AT, scale, AT, 1 << 40, None))


@pytest.mark.parametrize("args,want", [
    (dict(c=cache(head_dim=72)), api.ERR_INVALID), (dict(c=cache(reserved=1)), api.ERR_INVALID), (dict(q=heads(n=3)), api.ERR_MISMATCH),
    (dict(q=heads(data=None)), api.ERR_INVALID), (dict(prefix_table=None), api.ERR_INVALID), (dict(prefix_lengths=None), api.ERR_INVALID),
    (dict(starts=None), api.ERR_INVALID), (dict(prefix_stride=2), api.ERR_INVALID), (dict(prefix_stride=-3), api.ERR_INVALID),
    (dict(prefixes=1 << 31), api.ERR_INVALID), (dict(n=1 << 31), api.ERR_INVALID), (dict(scale=float("nan")), api.ERR_INVALID),
    (dict(scale=float("inf")), api.ERR_INVALID),
])
def test_shared_refusals(args, want):
    assert shared(**args) == want


def rows(data=AT, seq_stride=1000, row_stride=100, typ=BF16, reserved=0):
    return L.VocabRowsC(data, seq_stride, row_stride, typ, reserved)


@pytest.mark.parametrize("args,want", [
    (dict(seqs=(1 << 24) + 1), api.ERR_INVALID), (dict(n=65), api.ERR_INVALID), (dict(vocab=0), api.ERR_INVALID), (dict(vocab=(1 << 22) + 1), api.ERR_INVALID),
    (dict(target=None), api.ERR_INVALID), (dict(target=rows(data=None)), api.ERR_INVALID), (dict(target=rows(data=AT + 1)), api.ERR_INVALID),
    (dict(target=rows(typ=E4M3)), api.ERR_INVALID), (dict(target=rows(seq_stride=-1)), api.ERR_INVALID), (dict(target=rows(row_stride=(1 << 40) + 1)), api.ERR_INVALID),
    (dict(target=rows(reserved=1)), api.ERR_INVALID), (dict(draft=rows(typ=F16)), api.ERR_MISMATCH), (dict(draft=rows(data=None)), api.ERR_INVALID),
    (dict(drafts=None), api.ERR_INVALID), (dict(uniform=None), api.ERR_INVALID), (dict(tokens=None), api.ERR_INVALID), (dict(accepted=None), api.ERR_INVALID),
    (dict(temperature=AT, probabilities=1), api.ERR_INVALID),
])
def test_verify_refusals(args, want):
    a = dict(target=rows(), draft=rows(), seqs=3, n=4, vocab=100, drafts=AT, uniform=AT, temperature=None, probabilities=0, tokens=AT, accepted=AT)
    a.update(args)
    assert code(L.lib().bcp_verify_drafts(ref(a["target"]), ref(a["draft"]), *list(a.values())[2:], None)) == want


def test_no_sequences_is_no_error():
    assert L.lib().bcp_verify_drafts(None, None, 0, 4, 100, None, None, None, 0, None, None, None) == 0


def test_names_are_offered():
    for name in ("rope_axes", "bcp_kv_attend_shared", "bcp_verify_drafts"):
        assert callable(getattr(bcp, name)) and name in dir(bcp)
