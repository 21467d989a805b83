"""sp_cache_attention at the ends of what a call may say: texts beyond max_keys, logits beyond fp32, scales at the ends of their range."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api
from tests.test_gpu_paged_cache import filled, gen, ints, offsets, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_texts_beyond_max_keys_are_nan_whatever_their_length(four, causal):
    """The first chunk of a prompt (as many keys as queries), one with fewer keys than queries, one with more: reported, and NaN wherever a key is seen."""
    q_len, k_len, heads, kv, dh, page = [100, 120, 90, 90], [300, 120, 50, 200], 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 61)
    pages = filled(n_pages, kv, page, dh, four, 62)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(63), device=DEV).to(BF)
    cu = offsets(q_len)
    want, _ = api.sp_cache_attention(Q, pages, ints(cu), table, ints(k_len), heads, causal=causal, max_keys=sum(k_len))
    for left in range(len(k_len)):
        status = api.new_status()
        got, lse = api.sp_cache_attention(Q, pages, ints(cu), table, ints(k_len), heads, causal=causal, max_keys=sum(k_len[:left]) + k_len[left] - 1,
                                          want_lse=True, status=status)
        assert status.tolist()[0] == 2 and status.tolist()[1] >= left
        assert got[:cu[left]].isfinite().all()
        for s in range(left, len(k_len)):
            blind = max(0, q_len[s] - k_len[s]) if causal else 0             # queries before the first key
            assert (got[cu[s]:cu[s] + blind] == 0).all() and (lse[cu[s]:cu[s] + blind] == -math.inf).all()
            assert got[cu[s] + blind:cu[s + 1]].isnan().all() and lse[cu[s] + blind:cu[s + 1]].isnan().all()
    assert want.isfinite().all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("q_len, k_len", [([1, 2], [40, 700]), ([1], [30000]), ([300], [300])])
def test_scaled_logits_beyond_fp32_are_not_taken_for_a_mask(q_len, k_len, sign, dtype, four):
    """scale <q, k> = +-2^136 at every key: no probability can be told, so the rows are NaN, not 0, which says that a row sees no key."""
    heads, kv, dh, page = 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 64)
    pages = filled(n_pages, kv, page, dh, four, 65)
    if four:
        pages.k_scale[..., 0], pages.k_scale[..., 1] = 0.0, sign * 2.0 ** 66
    else:
        pages.k[:] = sign * 2.0 ** 66
    Q = torch.zeros(sum(q_len), heads * dh, dtype=dtype, device=DEV)
    Q[:, ::64] = 2.0 ** 60
    o, lse = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, scale=2.0 ** 10, want_lse=True)
    assert o.isnan().all() and not (lse == -math.inf).any()

@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [0.0, 1e-30, 1e-20])
@pytest.mark.parametrize("q_len, k_len", [([1, 2], [40, 701]), ([300], [300])])
def test_logits_too_small_for_fp32_are_equal(q_len, k_len, size, dtype, four):
    """Queries of (nearly) nothing times a scale of 1e-30: all keys that a query sees weigh the same."""
    heads, kv, dh, page = 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 66)
    pages = filled(n_pages, kv, page, dh, four, 67)
    Q = torch.full((sum(q_len), heads * dh), size, device=DEV).to(dtype)
    o, lse = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, scale=1e-30, want_lse=True)
    cu = offsets(q_len)
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        seen = torch.arange(nk - nq + 1, nk + 1, device=DEV).double()
        assert ((lse[cu[s]:cu[s + 1]].double() - seen.log()[:, None]).abs() <= 2.0 ** -18 * 10).all()
    assert o.isfinite().all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("where", [0, 15000, 29000])
def test_keys_of_no_weight_beside_others(where, dtype, four):
    """Logits of -2^136 at all keys but a thousand, whose logits are 0: the mean of their values, whichever pieces of the text hold them."""
    heads, kv, dh, page, n = 4, 2, 64, 16, 30000
    table, n_pages = table_for([n], page, 68)
    pages = filled(n_pages, kv, page, dh, four, 69)
    some = table[0, where // page:where // page + 62].long()
    if four:
        pages.k_scale[..., 0], pages.k_scale[..., 1] = 0.0, -2.0 ** 66
        pages.k_scale[some] = 0.0
    else:
        pages.k[:] = -2.0 ** 66
        pages.k[some] = 0.0
    Q = torch.zeros(1, heads * dh, dtype=dtype, device=DEV)
    Q[:, ::64] = 2.0 ** 60
    o, lse = api.sp_cache_attention(Q, pages, ints([0, 1]), table, ints([n]), heads, scale=2.0 ** 10, want_lse=True)
    from tests.test_gpu_paged_cache import values
    v = values(pages)[1][0][some].transpose(1, 2).flatten(0, 1)                   # [keys, kv, dh]
    want = v.mean(0).repeat_interleave(heads // kv, 0).flatten()
    assert ((lse.double() - math.log(v.shape[0])).abs() <= 1e-5).all()
    size = v.abs().mean(0).repeat_interleave(heads // kv, 0).flatten()
    assert ((o[0].double() - want).abs() <= (2.0 ** -8 if dtype == BF else 2.0 ** -20) * want.abs() + 2.0 ** (-11 if dtype == BF else -18) * 2 * size).all()


@pytest.mark.parametrize("q_len, k_len", [([1], [40]), ([1, 3], [5000, 33]), ([300], [500])])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_an_infinite_value_makes_its_channel_infinite(sign, q_len, k_len):
    """16 bits, bf16: at a key that all see, one that has the largest weight, and at the last one."""
    heads, kv, dh, page = 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 70)
    pages = filled(n_pages, kv, page, dh, False, 71)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(72), device=DEV).to(BF)
    for s, n in enumerate(k_len):
        for j, channel in ((0, 3), (n - 1, 5)):
            pages.v[int(table[s, j // page]), :, j % page, channel] = sign * math.inf
        pages.k[int(table[s, 0]), :, 0] = 0.0
    o, lse = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True)
    o = o.view(-1, heads, dh)
    assert (o[..., 3] == sign * math.inf).all() and lse.isfinite().all()
    last = [c - 1 for c in offsets(q_len)[1:]]
    assert (o[last][..., 5] == sign * math.inf).all()
    others = [c for c in range(dh) if c not in (3, 5)]
    assert o[..., others].isfinite().all()
