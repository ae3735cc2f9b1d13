"""Arguments of the attention over shared prefixes as its declaration allows them: workspaces anywhere on a 16-byte boundary, exactly as large as asked for; one row
of the prefixes' table for all groups."""
import pytest
import torch

import paper_2407_20143_b200 as bcp

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 64), (torch.float8_e4m3fn, 80), (torch.float16, 256)])
def test_workspaces_on_any_16_byte_boundary(cuda_device, dtype, dim):
    cache = bcp.KvCache.empty(40, 2, 16, dim, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((640, 2, dim), generator=g, device="cuda") for _ in range(2))
    bcp.bcp_kv_write(cache, k, v, torch.arange(640, device="cuda"))
    q = torch.randn((9, 8, dim), generator=g, device="cuda").to(torch.float16 if dtype == torch.float16 else torch.bfloat16)
    prefix_table, table = _int([list(range(30))]), _int([[30 + i] for i in range(9)])
    args = (prefix_table, _int([470]), _int([0, 7]), table, _int([9] * 9))
    want = bcp.bcp_kv_attend_shared(cache, q, *args)
    work = bcp.KvWorkspace(cache, 8, 9, shared=True)
    n, guard = work.bytes, 512
    for shift in (*range(0, 257, 16), 2032):
        memory = torch.zeros(2048 + n + guard, dtype=torch.uint8, device="cuda")
        memory[shift + n:] = 77
        work.memory, work.address = memory, memory.data_ptr() + shift
        assert work.address % 16 == 0
        for _ in range(2):
            out, lse = bcp.bcp_kv_attend_shared(cache, q, *args, workspace=work)
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            plain, _ = bcp.bcp_kv_attend(cache, q, table, args[4], workspace=work)
            assert torch.equal(plain, bcp.bcp_kv_attend(cache, q, table, args[4])[0])
        assert bool((memory[shift + n:] == 77).all()) and not memory[:shift].any()
    cache.check()


def test_a_workspace_that_is_too_small_or_off_the_boundary_is_refused(cuda_device):
    cache = bcp.KvCache.empty(4, 1, 16, 64, torch.bfloat16)
    q, table = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda"), _int([[1], [2], [3]])
    work = bcp.KvWorkspace(cache, 2, 3, shared=True)
    address, n = work.address, work.bytes
    call = lambda: bcp.bcp_kv_attend_shared(cache, q, _int([[0]]), _int([16]), _int([0, 3]), table, _int([5] * 3), workspace=work)  # noqa: E731
    call()
    for work.address, work.bytes in ((address + 8, n - 8), (address + 4, n - 4), (address + 16, n - 512)):
        with pytest.raises(bcp.BcpError):
            call()


@pytest.mark.parametrize("groups", [1, 2, 5])
def test_one_row_of_the_table_for_all_prefixes(cuda_device, groups):
    # prefixes of different lengths over the same pages
    cache = bcp.KvCache.empty(30, 2, 16, 64, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((480, 2, 64), generator=g, device="cuda") for _ in range(2))
    bcp.bcp_kv_write(cache, k, v, torch.arange(480, device="cuda"))
    q = torch.randn((10, 8, 64), generator=g, device="cuda").bfloat16()
    row = torch.randperm(20, generator=torch.Generator().manual_seed(1)).int().cuda()[None]
    lengths, starts = _int([320 - 37 * i for i in range(groups)]), _int([10 * i // groups for i in range(groups + 1)])
    more = (lengths, starts, _int([[20 + i] for i in range(10)]), _int([7] * 10))
    expanded = row.expand(groups, -1)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, expanded, *more)
    want, sums = bcp.bcp_kv_attend_shared(cache, q, expanded.contiguous(), *more)
    cache.check()
    assert torch.equal(out, want) and torch.equal(lse, sums)
