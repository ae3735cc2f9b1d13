"""What becomes of a call of the attention over shared prefixes whose waits run out: it ends, says so in the cache's status word, and leaves its workspace
ready for the next call.  With a limit of zero waits of a sound call pass it."""
import pytest
import torch

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import _lib as L
from paper_2407_20143_b200 import api, decode

pytestmark = pytest.mark.gpu

TWO_SECONDS = 2_000_000_000


@pytest.fixture
def limit():
    yield L.lib().bcp_wait_limit
    assert L.lib().bcp_wait_limit(TWO_SECONDS) == 0


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("dim,seqs,page", [(128, 70, 64), (64, 9, 7), (256, 20, 16), (128, 3, 24)])
def test_waits_that_run_out_end_the_call(cuda_device, limit, dtype, dim, seqs, page):
    n = 6000 // page
    cache = bcp.KvCache.empty(n + seqs, 2, page, dim, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(((n + seqs) * page, 2, dim), generator=g, device="cuda") for _ in range(2))
    bcp.bcp_kv_write(cache, k, v, torch.arange((n + seqs) * page, device="cuda"))
    q = torch.randn((seqs, 16, dim), generator=g, device="cuda").to(torch.float16 if dtype == torch.float16 else torch.bfloat16)
    third, half = n // 3, seqs // 2
    prefix_table = _int([list(range(n)), [*range(third), *[0] * (n - third)]])
    args = (prefix_table, _int([n * page, third * page - 3]), _int([0, half, seqs]), _int([[n + i] for i in range(seqs)]), _int([5] * seqs))
    work = bcp.KvWorkspace(cache, 16, seqs, shared=True)
    want = bcp.bcp_kv_attend_shared(cache, q, *args, workspace=work)
    cache.check()
    ran_out = 0
    for ns in [0] * 12:
        assert limit(ns) == 0
        bcp.bcp_kv_attend_shared(cache, q, *args, workspace=work)
        assert limit(TWO_SECONDS) == 0
        try:
            cache.check()
        except bcp.BcpError as e:
            assert e.code == api.ERR_BOUNDS and "ran out" in str(e)
            ran_out += 1
        out, lse = bcp.bcp_kv_attend_shared(cache, q, *args, workspace=work)
        cache.check()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert ran_out > 0


def test_what_the_status_word_is_reported_as(cuda_device):
    cache = bcp.KvCache.empty(1, 1, 16, 64)
    outside = "an index was outside its range and was left out:"
    for bits, says, not_says in ((decode.TIMED_OUT, ["a wait", "ran out"], [outside]), (decode.BAD_PAGE, [outside + " page"], ["wait", "slot"]),
                                 (decode.TIMED_OUT | decode.BAD_LENGTH | decode.BAD_SLOT, ["a wait", "ran out", outside + " slot length"], ["page"])):
        cache.status.fill_(bits)
        with pytest.raises(bcp.BcpError) as e:
            cache.check()
        assert e.value.code == api.ERR_BOUNDS and all(x in str(e.value) for x in says) and not any(x in str(e.value) for x in not_says)
        cache.check()
