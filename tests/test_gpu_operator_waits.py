"""A wait inside the attention kernels that runs out ends the call with SP_ERR_TIMEOUT in the status word; the context stays usable, and
the next call is right.  (The budget is cut to a few cycles.  The instruction that waits may itself hold a thread for a while before the clock
is read, so an ordinary wait may still end in time: then the call has to be right.)"""
import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("q,k", [([300, 40], [300, 90]), ([1, 1], [3000, 70])])      # tiles of many rows; single tokens
def test_waits_that_run_out(q, k):
    heads, dh = 8, 64
    cu = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=DEV)
    Q, K, V = (torch.randn(sum(n), heads * dh, device=DEV).bfloat16() for n in (q, k, k))
    want, _ = api.sp_attention(Q, K, V, cu(q), cu(k), heads)
    status = api.new_status()
    torch.cuda.synchronize()
    api._check(api.lib().sp_set_wait_budget(8), "sp_set_wait_budget")
    try:
        for _ in range(4):
            status.zero_()
            got, _ = api.sp_attention(Q, K, V, cu(q), cu(k), heads, status=status)
            torch.cuda.synchronize()
            assert int(status[0]) in (0, 7)
            assert int(status[0]) == 7 or torch.equal(got, want)
    finally:
        api._check(api.lib().sp_set_wait_budget(0), "sp_set_wait_budget")
    status.zero_()
    got, _ = api.sp_attention(Q, K, V, cu(q), cu(k), heads, status=status)
    assert torch.equal(got, want) and int(status[0]) == 0


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("q,k,role", [([4096], [4096], (11, 12, 13, 14)), ([1] * 16, [8000] * 16, (21,))])
def test_every_form_gives_up_a_wait(dh, q, k, role):
    """Calls of many key tiles for every SM: some wait is for a copy or a product that has only begun, and the call ends with SP_ERR_TIMEOUT
    from one of its form's roles."""
    heads = 8
    cu = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(dh)
    Q, K, V = (torch.randn(sum(n), heads * dh, generator=g, device=DEV).bfloat16() for n in (q, k, k))
    cq, ck, status = cu(q), cu(k), api.new_status()
    want, _ = api.sp_attention(Q, K, V, cq, ck, heads, status=status)
    assert status.tolist() == [0, 0, 0, 0]
    api._check(api.lib().sp_set_wait_budget(8), "sp_set_wait_budget")
    try:
        for _ in range(3):
            status.zero_()
            api.sp_attention(Q, K, V, cq, ck, heads, status=status)
            torch.cuda.synchronize()
            assert int(status[0]) == 7 and int(status[2]) in role
    finally:
        api._check(api.lib().sp_set_wait_budget(0), "sp_set_wait_budget")
    status.zero_()
    got, _ = api.sp_attention(Q, K, V, cq, ck, heads, status=status)
    assert torch.equal(got, want) and status.tolist() == [0, 0, 0, 0]
