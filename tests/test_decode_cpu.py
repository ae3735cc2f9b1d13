"""Host side of the decoding operators: descriptors, refusals (all of them before anything touches a GPU), the frequencies of
the rotation tables.  The addresses below are made up; every call must be refused before it could use one."""
import ctypes as C
import math

import pytest

from paper_2407_20143_b200 import _lib as L
from paper_2407_20143_b200 import api

AT = 1 << 20  # a made-up address, aligned to everything
BF16, F16, F32, E4M3, I8 = 2, 3, 1, 4, 5


def heads(n=2, token_stride=128, head_stride=64, typ=BF16, data=AT):
    return L.HeadsC(data, token_stride, head_stride, n, typ)


def table(**k):
    a = dict(table=AT, n_positions=100, rot_dim=64, layout=0, status=None)
    a.update(k)
    return L.RopeTableC(*a.values())


def cache(**k):
    a = dict(k=AT, v=AT, k_scale=None, v_scale=None, page_stride=2048, head_stride=1024, token_stride=64, n_pages=4, page_size=16, n_heads=2,
             head_dim=64, format=BF16, reserved=0, status=None)
    a.update(k)
    return L.KvCacheC(*a.values())


def code(rc):
    assert rc < 0 and L.lib().bcp_last_error()
    return rc


def rope(q=None, out=None, k=None, k_out=None, dim=64, tokens=4, tab=None, positions=AT):
    q, out, tab = q or heads(), out or heads(), tab or table()
    ref = lambda x: C.addressof(x) if x is not None else None  # noqa: E731
    return code(L.lib().bcp_rope(ref(q), ref(out), ref(k), ref(k_out), dim, tokens, ref(tab), positions, 0, None))


def test_descriptor_sizes():
    assert C.sizeof(L.HeadsC) == 32 and C.sizeof(L.RopeTableC) == 32 and C.sizeof(L.KvCacheC) == 88


@pytest.mark.parametrize("args,want", [
    (dict(dim=1), api.ERR_INVALID), (dict(dim=257), api.ERR_INVALID), (dict(tokens=-1), api.ERR_INVALID), (dict(tokens=1 << 31), api.ERR_INVALID),
    (dict(positions=None), api.ERR_INVALID), (dict(tab=table(rot_dim=66)), api.ERR_INVALID), (dict(tab=table(rot_dim=7)), api.ERR_INVALID),
    (dict(tab=table(rot_dim=0)), api.ERR_INVALID), (dict(tab=table(layout=2)), api.ERR_INVALID), (dict(tab=table(table=None)), api.ERR_INVALID),
    (dict(tab=table(table=AT + 4)), api.ERR_INVALID), (dict(tab=table(n_positions=0)), api.ERR_INVALID),
    (dict(q=heads(typ=E4M3)), api.ERR_INVALID), (dict(q=heads(typ=0)), api.ERR_INVALID), (dict(q=heads(data=None)), api.ERR_INVALID),
    (dict(q=heads(data=AT + 1)), api.ERR_INVALID), (dict(q=heads(n=0)), api.ERR_INVALID), (dict(q=heads(token_stride=-128)), api.ERR_INVALID),
    (dict(q=heads(token_stride=1 << 32)), api.ERR_INVALID), (dict(out=heads(typ=F32)), api.ERR_MISMATCH), (dict(out=heads(n=1)), api.ERR_MISMATCH),
    (dict(out=heads(token_stride=64)), api.ERR_DST_ALIAS), (dict(out=heads(head_stride=0)), api.ERR_DST_ALIAS),
    (dict(out=heads(head_stride=63)), api.ERR_DST_ALIAS), (dict(k=heads()), api.ERR_INVALID), (dict(k_out=heads()), api.ERR_INVALID),
    (dict(k=heads(typ=F16), k_out=heads(typ=F16)), api.ERR_MISMATCH),
])
def test_rope_refusals(args, want):
    assert rope(**args) == want


BAD_CACHES = [
    (dict(format=F32), api.ERR_INVALID), (dict(format=9), api.ERR_INVALID), (dict(reserved=1), api.ERR_INVALID), (dict(head_dim=0), api.ERR_INVALID),
    (dict(head_dim=72), api.ERR_INVALID), (dict(head_dim=272), api.ERR_INVALID), (dict(n_heads=0), api.ERR_INVALID), (dict(page_size=0), api.ERR_INVALID),
    (dict(n_pages=0), api.ERR_INVALID), (dict(n_pages=1 << 28), api.ERR_INVALID), (dict(k=None), api.ERR_INVALID), (dict(v=AT + 8), api.ERR_INVALID),
    (dict(page_stride=0), api.ERR_INVALID), (dict(token_stride=-64), api.ERR_INVALID), (dict(token_stride=68), api.ERR_INVALID),
    (dict(page_stride=1 << 32), api.ERR_INVALID), (dict(format=E4M3), api.ERR_INVALID), (dict(k_scale=AT, v_scale=AT), api.ERR_INVALID),
    (dict(format=I8, k_scale=AT, v_scale=AT + 2), api.ERR_INVALID), (dict(token_stride=32), api.ERR_DST_ALIAS), (dict(head_stride=512), api.ERR_DST_ALIAS),
    (dict(page_stride=1024), api.ERR_DST_ALIAS),
]


@pytest.mark.parametrize("args,want", BAD_CACHES)
def test_cache_refusals(args, want):
    c, h = cache(**args), heads()
    assert code(L.lib().bcp_kv_write(C.addressof(c), C.addressof(h), C.addressof(h), AT, 4, None, None, None)) == want
    assert code(L.lib().bcp_kv_read(C.addressof(c), AT, 4, C.addressof(h), C.addressof(h), None)) == want
    assert code(L.lib().bcp_kv_attend(C.addressof(c), C.addressof(h), C.addressof(h), AT, 4, AT, 3, 3, AT, 1.0, 0, AT, 1 << 40, None)) == want
    n = C.c_uint64()
    assert code(L.lib().bcp_kv_attend_workspace(C.addressof(c), 2, 4, C.byref(n))) == want


def test_layouts_of_the_cache_that_do_not_overlap_are_told_from_those_that_do():
    # tokens before heads, keys and values of a page side by side, heads outermost: refused only for their missing slots
    for k in (dict(token_stride=128, head_stride=64), dict(page_stride=4096), dict(head_stride=4096, page_stride=1024)):
        c, h = cache(**k), heads()
        assert code(L.lib().bcp_kv_write(C.addressof(c), C.addressof(h), C.addressof(h), None, 4, None, None, None)) == api.ERR_INVALID
        assert b"slots" in L.lib().bcp_last_error()


@pytest.mark.parametrize("k,v,want", [(heads(n=3, token_stride=192), heads(n=3, token_stride=192), api.ERR_MISMATCH), (heads(), heads(typ=F16), api.ERR_MISMATCH),
                                      (heads(), heads(n=1), api.ERR_MISMATCH), (heads(typ=I8), heads(), api.ERR_INVALID)])
def test_write_and_read_refusals(k, v, want):
    c = cache()
    assert code(L.lib().bcp_kv_write(C.addressof(c), C.addressof(k), C.addressof(v), AT, 4, None, None, None)) == want
    assert code(L.lib().bcp_kv_read(C.addressof(c), AT, 4, C.addressof(k), C.addressof(v), None)) == want
    t = table(rot_dim=128)
    h = heads()
    assert code(L.lib().bcp_kv_write(C.addressof(c), C.addressof(h), C.addressof(h), AT, 4, C.addressof(t), AT, None)) == api.ERR_INVALID
    t = table()
    assert code(L.lib().bcp_kv_write(C.addressof(c), C.addressof(h), C.addressof(h), AT, 4, C.addressof(t), None, None)) == api.ERR_INVALID
    assert code(L.lib().bcp_kv_read(C.addressof(c), AT, 4, C.addressof(heads(token_stride=0)), C.addressof(h), None)) == api.ERR_DST_ALIAS


def attend(c=None, q=None, out=None, n=4, blocks=AT, stride=3, width=3, lengths=AT, scale=1.0):
    c, q, out = c or cache(), q or heads(), out or heads()
    return code(L.lib().bcp_kv_attend(C.addressof(c), C.addressof(q), C.addressof(out), AT, n, blocks, stride, width, lengths, scale, 0, AT, 1 << 40, None))


@pytest.mark.parametrize("args,want", [
    (dict(q=heads(n=3, token_stride=192), out=heads(n=3, token_stride=192)), api.ERR_MISMATCH), (dict(q=heads(n=4, token_stride=256)), api.ERR_MISMATCH),
    (dict(q=heads(typ=F16), out=heads(typ=F16)), api.ERR_MISMATCH), (dict(out=heads(typ=F16)), api.ERR_MISMATCH),
    (dict(c=cache(format=E4M3, k_scale=AT, v_scale=AT), q=heads(typ=F32), out=heads(typ=F32)), api.ERR_MISMATCH),
    (dict(q=heads(data=AT + 4)), api.ERR_INVALID), (dict(q=heads(token_stride=130)), api.ERR_INVALID), (dict(out=heads(data=AT + 2)), api.ERR_INVALID),
    (dict(blocks=None), api.ERR_INVALID), (dict(lengths=None), api.ERR_INVALID), (dict(stride=2), api.ERR_INVALID), (dict(stride=-3), api.ERR_INVALID),
    (dict(scale=math.nan), api.ERR_INVALID), (dict(scale=math.inf), api.ERR_INVALID), (dict(out=heads(token_stride=0)), api.ERR_DST_ALIAS),
])
def test_attend_refusals(args, want):
    assert attend(**args) == want


def test_status_needs_a_word():
    assert code(L.lib().bcp_decode_status(None, None)) == api.ERR_INVALID


def test_frequencies():
    import paper_2407_20143_b200 as bcp

    f = bcp.rope_frequencies(8, base=100.0)
    assert f == pytest.approx([1.0, 100 ** -0.25, 0.1, 100 ** -0.75])
    assert bcp.rope_frequencies(8, base=100.0, scaling="linear", factor=4.0) == pytest.approx([x / 4 for x in f])
    b = bcp.rope_frequencies(8, base=100.0, scaling="base", factor=4.0)
    assert b[0] == 1.0 and b[-1] == pytest.approx(f[-1] / 4) and all(x <= y for x, y in zip(b, f))
    # over 40 tokens the four pairs turn 6.4, 2.0, 0.64 and 0.2 times: kept, mixed, and two divided
    s = bcp.rope_frequencies(8, base=100.0, scaling="bands", factor=8.0, trained=40)
    keep = (40 * f[1] / (2 * math.pi) - 1) / 3
    assert s == pytest.approx([f[0], f[1] * keep + f[1] / 8 * (1 - keep), f[2] / 8, f[3] / 8])
    for bad in (lambda: bcp.rope_frequencies(7), lambda: bcp.rope_frequencies(8, scaling="other"), lambda: bcp.rope_frequencies(8, factor=0.5),
                lambda: bcp.rope_frequencies(8, scaling="bands", factor=2.0), lambda: bcp.rope_frequencies(8, base=0.0)):
        with pytest.raises(bcp.BcpError):
            bad()


def test_tensors_on_the_cpu_are_refused():
    import torch

    import paper_2407_20143_b200 as bcp

    with pytest.raises(bcp.BcpError):
        bcp.RopeTable(torch.zeros(4, 2, 8))
    with pytest.raises(bcp.BcpError):
        bcp.KvCache(torch.zeros(2, 2, 4, 32, dtype=torch.bfloat16), torch.zeros(2, 2, 4, 32, dtype=torch.bfloat16))


def test_the_host_only_calls_do_not_import_torch():
    import subprocess
    import sys

    code_ = "import sys, paper_2407_20143_b200 as b; b.bcp_decompose((4, 4), 1, 5); assert 'torch' not in sys.modules; print('ok')"
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code_], capture_output=True, text=True, cwd=root, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr


def slots(table, sequences, positions, n_pages=12, page_size=16):
    from types import SimpleNamespace

    import torch

    from paper_2407_20143_b200 import decode

    row = lambda x: x if isinstance(x, int) else torch.tensor(x, dtype=torch.int64)  # noqa: E731
    got = decode.KvCache.slots(SimpleNamespace(n_pages=n_pages, page_size=page_size), torch.tensor(table, dtype=torch.int32), row(sequences), row(positions))
    assert got.dtype == torch.int64
    return got.tolist()


def test_slots_of_tokens():
    table = [[5, 9], [3, -1]]
    assert slots(table, [0, 0, 0, 1, 1], [0, 15, 16, 7, 15]) == [80, 95, 144, 55, 63]
    assert slots(table, 1, [0, 3]) == [48, 51]  # one row for all
    assert slots(table, [0, 0], [6, 7], page_size=7) == [41, 63]


def test_slots_of_padding_are_skipped():
    # position -1 marks padding everywhere else; it must not become the last slot of the last page
    assert slots([[5, 9]], [0, 0, 0], [-1, -16, -(1 << 40)]) == [-1, -1, -1]
    # a page that the table does not have yet
    assert slots([[5, -1], [-7, 2]], [0, 1, 1], [17, 15, 16]) == [-1, -1, 32]


def test_slots_past_the_table_are_past_the_cache():
    # so that the write or read reports them (a plain index past the table's end would stop the whole GPU context)
    assert slots([[5, 9], [5, -1]], [0, 1, 0], [32, 32, 1 << 40]) == [12 * 16] * 3
    assert slots([[5, 9]], [1, -1, 0], [0, 0, 0]) == [12 * 16, 12 * 16, 80]
    assert slots([[5, 9]], [1, 7], [-1, -1]) == [-1, -1]
    assert slots([[]], [0, 0], [0, -1]) == [12 * 16, -1]


def test_slots_of_any_index_type():
    from types import SimpleNamespace

    import torch

    from paper_2407_20143_b200 import decode

    big = SimpleNamespace(n_pages=1 << 20, page_size=1 << 10)  # slots up to 2^30, products of int32 past 2^31
    table = torch.tensor([[(1 << 20) - 1, 4]], dtype=torch.int32)
    for typ in (torch.int32, torch.int64):
        got = decode.KvCache.slots(big, table, torch.tensor([0, 0, 0], dtype=typ), torch.tensor([5, 1024, 2048], dtype=typ))
        assert got.dtype == torch.int64 and got.tolist() == [((1 << 20) - 1) * 1024 + 5, 4096, 1 << 30]
    assert decode.KvCache.slots(big, table.expand(3, 2), [2, 1], torch.tensor([7, 1025])).tolist() == [((1 << 20) - 1) * 1024 + 7, 4097]
    with pytest.raises(IndexError):
        decode.KvCache.slots(big, table, 1, torch.tensor([5]))


def run_without_torch(code_):
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", "import sys; sys.modules['torch'] = None\n" + code_], capture_output=True, text=True, cwd=root, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr


def test_a_star_import_needs_no_torch():
    run_without_torch("from paper_2407_20143_b200 import *\nassert bcp_decompose((4, 4), 1, 5) and bcp_plan and Plan; print('ok')")


def test_the_lazy_names_are_listed_and_found():
    import paper_2407_20143_b200 as bcp

    names = {"KvCache", "KvWorkspace", "RopeTable", "bcp_kv_attend", "bcp_kv_read", "bcp_kv_write", "bcp_rope", "bcp_rope_backward", "rope", "rope_frequencies"}
    assert names <= set(dir(bcp)) and all(callable(getattr(bcp, n)) for n in names)
    with pytest.raises(AttributeError):
        bcp.no_such_name


def test_the_library_is_built_without_torch():
    run_without_torch("""
from paper_2407_20143_b200 import build
build.build_library = lambda force=False, verbose=False: "library"
build.build_binding = lambda force=False: 1 / 0
assert build.build_all(force=True) == ["library"]; print('ok')""")


def test_all_is_built_with_torch(monkeypatch):
    from paper_2407_20143_b200 import build

    monkeypatch.setattr(build, "build_library", lambda force=False, verbose=False: "library")
    monkeypatch.setattr(build, "build_binding", lambda force=False: "binding")
    assert build.build_all() == ["library", "binding"]
