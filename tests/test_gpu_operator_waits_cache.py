"""A wait that runs out inside the 8-bit product and inside the tiles over an opened cache ends the call with SP_ERR_TIMEOUT in the status word; the
context stays usable, and the next call is right.  (The budget is cut to a few cycles, for calls of many tiles for every SM: some wait is for a copy or a
product that has only begun.)"""
import pytest
import torch

from paper_2510_03246_b200 import api
from tests.test_gpu_paged_cache import filled, gen, ints, offsets, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F8 = torch.bfloat16, torch.float8_e4m3fn


def short_waits(call, want, same):
    status = api.new_status()
    torch.cuda.synchronize()
    api._check(api.lib().sp_set_wait_budget(8), "sp_set_wait_budget")
    try:
        for _ in range(3):
            status.zero_()
            call(status)
            torch.cuda.synchronize()
            assert int(status[0]) == 7
    finally:
        api._check(api.lib().sp_set_wait_budget(0), "sp_set_wait_budget")
    status.zero_()
    assert same(call(status), want) and status.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("T, n_in, n_out", [(4096, 4096, 4096), (2048, 2000, 3303)])
def test_8_bit_products_give_up_a_wait(T, n_in, n_out):
    X, W = (api.rows_of_16_bytes(n, n_in, F8, DEV) for n in (T, n_out))
    for m, seed in ((X, 1), (W, 2)):
        m.copy_(torch.randn(m.shape, generator=gen(seed), device=DEV))
    xs, ws = torch.ones(T, device=DEV), torch.full((n_out,), n_in ** -0.5, device=DEV)
    want = api.sp_linear_e4m3(X, xs, W, ws)
    short_waits(lambda status: api.sp_linear_e4m3(X, xs, W, ws, status=status), want, torch.equal)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_tiles_over_a_cache_give_up_a_wait(four, dh):
    q_len, k_len, heads, kv, page = [2048], [8192], 8, 4, 64
    table, n_pages = table_for(k_len, page, 71)
    pages = filled(n_pages, kv, page, dh, four, 72)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(73), device=DEV).to(BF)

    def call(status):
        return api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, max_keys=sum(k_len), status=status)[0]

    short_waits(call, call(None), torch.equal)
