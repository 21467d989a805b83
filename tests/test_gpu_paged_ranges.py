"""sp_cache_attention over 4-bit pages whose values have very different sizes: what another text, another head, another query or a key that a query
does not see holds costs its result nothing.

Tolerances count roundings.  fp16 is off by 2^-11 of a value at most, bf16 by 2^-8, sums in fp32 by 2^-19 of their terms' sizes (128 channels, and the
partial sums of a tile).  With many rows keys are opened in one rounding, a query's values are exact; probabilities and opened values have one rounding each.  With few
rows a query's values may lose 2^-16 of the row's largest, the numbers are exact, probabilities times scales have one rounding.  The result has half a step of bf16."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api
from tests.test_gpu_paged_cache import filled, gathered, gen, ints, offsets, table_for, values

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def copied(pages):
    return api.KvPages(*(None if x is None else x.clone() for x in (pages.k, pages.v, pages.k_scale, pages.v_scale)))


def call(Q, pages, q_len, table, k_len, heads, **kw):
    status = api.new_status()
    out, lse = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True, status=status, **kw)
    assert status.tolist() == [0, 0, 0, 0]
    return out, lse


def within(got, lse, Q, pages, q_len, table, k_len, heads, page, rounding, few, rows=None):
    """Every value (of rows and heads [Nq, n_heads]) against the formula in 64 bits.  rounding: of probabilities and opened values."""
    kv = pages.k.shape[1]
    (k64, k_size), (v64, v_size) = values(pages)
    dh, g, cu = k64.shape[3], heads // kv, offsets(q_len)
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        if nq == 0:
            continue
        q = Q[cu[s]:cu[s + 1]].double().view(nq, kv, g, dh)
        K, V, KS, VS = (gathered(x, table, page, s, nk) for x in (k64, v64, k_size, v_size))
        hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq
        z = (torch.einsum("iagd,jad->agij", q, K) * dh ** -0.5).masked_fill(hidden, -math.inf)
        size = torch.einsum("iagd,jad->agij", q.abs(), KS) * 2.0 ** -19
        if few:
            size = size + torch.einsum("iag,ja->agij", q.abs().amax(3), KS.sum(2)) * 2.0 ** -16
        else:
            size = size + torch.einsum("iagd,jad->agij", q.abs(), K.abs()) * rounding
        size = (size * dh ** -0.5).masked_fill(hidden, 0.0)
        want_lse = torch.logsumexp(z, 3)
        p = torch.where(want_lse[..., None] == -math.inf, 0.0, (z - want_lse[..., None]).exp())
        want = torch.einsum("agij,jad->iagd", p, V)
        moved = torch.expm1(size.clamp(max=1.0)) + torch.expm1((p * size).sum(3).clamp(max=1.0))[..., None]
        off = torch.einsum("agij,jad->iagd", p * (moved + 2.0 ** -19 + rounding * (1 if few else 2)), VS) + 2.0 ** -8 * want.abs() + 1e-7
        o = got[cu[s]:cu[s + 1]].double().view(nq, kv, g, dh)
        of = torch.ones(nq, heads, dtype=torch.bool, device=DEV) if rows is None else rows[cu[s]:cu[s + 1]]
        of = of.view(nq, kv, g)
        assert ((o - want).abs() <= off)[of].all(), (s, ((o - want).abs() / off)[of].max().item())
        have = lse[cu[s]:cu[s + 1]].double().view(nq, kv, g).permute(1, 2, 0)
        of, none = of.permute(1, 2, 0), want_lse == -math.inf
        assert torch.equal((have == -math.inf)[of], none[of])
        assert ((have - want_lse).abs() <= size.amax(3) + 2.0 ** -19 * (1 + want_lse.abs()))[~none & of].all()


FORMS = {"few": ([4, 1], [200, 90]), "many": ([140, 100], [400, 130])}


def setup(rows, seed, heads=4, kv=2, dh=128, page=16):
    q_len, k_len = FORMS[rows]
    table, n_pages = table_for(k_len, page, seed)
    pages = filled(n_pages, kv, page, dh, True, seed + 1)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(seed + 2), device=DEV).to(BF)
    return q_len, k_len, table, pages, Q, heads, page


def at(table, s, j, page):
    return int(table[s, j // page]), j % page


@pytest.mark.parametrize("size", [1e9, 1e30])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_another_text(rows, which, size):
    """A large scale, a large offset of another text: not a bit."""
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 1)
    want, lse = call(Q, pages, q_len, table, k_len, heads)
    within(want, lse, Q, pages, q_len, table, k_len, heads, page, 2.0 ** -11, rows == "few")
    for entry in (0, 1):
        bad = copied(pages)
        pg, slot = at(table, 1, 20, page)
        (bad.k_scale if which == "k" else bad.v_scale)[pg, :, slot, 0, entry] = size
        got, other = call(Q, bad, q_len, table, k_len, heads)
        assert torch.equal(got[:q_len[0]], want[:q_len[0]]) and torch.equal(other[:q_len[0]], lse[:q_len[0]])


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_another_head(rows, which):
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 4)
    want, lse = call(Q, pages, q_len, table, k_len, heads)
    bad = copied(pages)
    for s in (0, 1):
        pg, slot = at(table, s, 33, page)
        (bad.k_scale if which == "k" else bad.v_scale)[pg, 1, slot] = 1e30
    got, other = call(Q, bad, q_len, table, k_len, heads)
    half = want.shape[1] // 2                                    # (the query heads of key head 0)
    assert torch.equal(got[:, :half], want[:, :half]) and torch.equal(other[:, :heads // 2], lse[:, :heads // 2])


@pytest.mark.parametrize("rows", ["few", "many"])
def test_another_query(rows):
    """Not a bit where a row has its own units and reference (many rows); the references of a tile of few rows rise together."""
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 7)
    want, lse = call(Q, pages, q_len, table, k_len, heads)
    big, dh = Q.clone(), Q.shape[1] // heads
    big[2] *= 1e20
    big[1, dh:2 * dh] = 1e25
    got, other = call(big, pages, q_len, table, k_len, heads)
    same = torch.ones(Q.shape[0], heads, dtype=torch.bool, device=DEV)
    same[2], same[1, 1] = False, False
    within(got, other, big, pages, q_len, table, k_len, heads, page, 2.0 ** -11, rows == "few", same)
    if rows == "many":
        assert torch.equal(got.view(-1, heads, dh)[same], want.view(-1, heads, dh)[same]) and torch.equal(other[same], lse[same])


@pytest.mark.parametrize("size", [300.0, 1e9, 1e30])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_a_key_that_only_later_queries_see(rows, which, size):
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 10)
    bad = copied(pages)
    key = k_len[0] - 1
    pg, slot = at(table, 0, key, page)
    (bad.k_scale if which == "k" else bad.v_scale)[pg, :, slot, :, 0] = size
    got, lse = call(Q, bad, q_len, table, k_len, heads)
    # all but the last query of the first text, which alone sees the key
    n = q_len[0] - 1
    keep = [i for i in range(sum(q_len)) if i != n]
    within(got[keep], lse[keep], Q[keep], bad, [n, q_len[1]], table, [k_len[0] - 1, k_len[1]], heads, page, 2.0 ** -11 if size < 1e6 else 2.0 ** -8, rows == "few")
    assert got[n].isfinite().all() or size > 1e6                # (logits beyond 2^31 leave its own exponents nothing)


@pytest.mark.parametrize("rows", ["few", "many"])
@pytest.mark.parametrize("far", [2.0 ** 19, 2.0 ** 24, 2.0 ** 60])
def test_a_large_value_of_no_weight(rows, far):
    """A key whose probability vanishes may hold values of any size: the others keep theirs.  (Offsets: K of the key is far below, so that its logit is.)"""
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 13)
    Q = Q.abs()
    bad = copied(pages)
    for s in (0, 1):
        pg, slot = at(table, s, 5, page)
        bad.k_scale[pg, :, slot, :, 1] = -40.0                   # logits of -40 sum |q| / sqrt 128: some -350
        bad.v_scale[pg, :, slot] *= far
    got, lse = call(Q, bad, q_len, table, k_len, heads)
    within(got, lse, Q, bad, q_len, table, k_len, heads, page, 2.0 ** -8, rows == "few")


@pytest.mark.parametrize("rows", ["few", "many"])
@pytest.mark.parametrize("by", [2.0 ** -30, 2.0 ** 30, 2.0 ** 90])
def test_values_that_change_by_steps(rows, by):
    """The scales of V change once on the way, so far that no unit holds both sides, and one group of 64 channels differs from the other."""
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 16)
    bad = copied(pages)
    for s in (0, 1):
        for j in range(k_len[s] // 2, k_len[s]):
            pg, slot = at(table, s, j, page)
            bad.v_scale[pg, 0, slot] *= by
            bad.v_scale[pg, 1, slot, 1] *= by
    got, lse = call(Q, bad, q_len, table, k_len, heads)
    within(got, lse, Q, bad, q_len, table, k_len, heads, page, 2.0 ** -8 if rows == "many" else 2.0 ** -11, rows == "few")


def test_many_long_texts_each_with_values_of_its_own_size():
    """More rows than the blocks that look for the sizes take at once, texts that end inside a warp's rows and behind them."""
    q_len, k_len, heads, kv, dh, page = [40] * 13, [2048 + 37 * i for i in range(12)] + [41], 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 19)
    pages = filled(n_pages, kv, page, dh, True, 20)
    for s, n in enumerate(k_len):                                # 2^-50 .. 2^55 for V, beside 1 for K
        pg = table[s, :-(-n // page)].long()
        pages.v_scale[pg] *= 2.0 ** (-50 + 8 * s + s % 2)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(21), device=DEV).to(BF)
    got, lse = call(Q, pages, q_len, table, k_len, heads, max_keys=sum(k_len))
    cu = offsets(q_len)
    for s, n in enumerate(k_len):
        back = copied(pages)
        back.v_scale[table[s, :-(-n // page)].long()] *= 2.0 ** (50 - 8 * s - s % 2)
        rows = slice(cu[s], cu[s + 1])
        within(got[rows] * 2.0 ** (50 - 8 * s - s % 2), lse[rows], Q[rows], back, q_len[s:s + 1], table[s:s + 1], [n], heads, page, 2.0 ** -11, False)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads, kv, q_len, k_len", [(8, 2, [4, 3], [200, 90]), (4, 4, [1, 1], [700, 33]), (16, 1, [1], [3000]), (3, 1, [5, 1, 2], [60, 9000, 17])])
@pytest.mark.parametrize("by", [2.0 ** 30, 2.0 ** -40])
def test_few_rows_of_every_tile_and_width(by, heads, kv, q_len, k_len, dh):
    """Scales of V that change by steps in every third block, pieces of a long text that meet them and others that do not."""
    page = 16
    table, n_pages = table_for(k_len, page, 22)
    pages = filled(n_pages, kv, page, dh, True, 23)
    for s, n in enumerate(k_len):
        for e in range(1, -(-n // page), 3):
            pages.v_scale[int(table[s, e]), :, ::5] *= by
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(24), device=DEV).to(BF)
    got, lse = call(Q, pages, q_len, table, k_len, heads)
    within(got, lse, Q, pages, q_len, table, k_len, heads, page, 2.0 ** -11, True)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads, kv", [(4, 4), (70, 1)])
def test_formats_of_items_side_by_side(heads, kv, dh):
    """More items than SMs, fp16 and bf16 in turn; heads of a group that go one by one (more than 64 share a key head)."""
    n, page = (60, 16) if kv == 4 else (12, 16)
    q_len, k_len = [64 if kv == 4 else 40] * n, [65 + 17 * (i % 20) for i in range(n)]
    table, n_pages = table_for(k_len, page, 25)
    pages = filled(n_pages, kv, page, dh, True, 26)
    wide = torch.zeros(n, kv, dtype=torch.bool)
    for s in range(n):
        for h in range(kv):
            if (s + h) % 3 == 0:
                wide[s, h] = True
                pages.v_scale[int(table[s, 1]), h, 3] *= 2.0 ** 26
                if (s + h) % 2:
                    pages.k_scale[int(table[s, 0]), h, 7] *= 2.0 ** -24
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(27), device=DEV).to(BF)
    got, lse = call(Q, pages, q_len, table, k_len, heads, max_keys=sum(k_len))
    rows = wide.repeat_interleave(heads // kv, 1).repeat_interleave(torch.tensor(q_len), 0).to(DEV)
    within(got, lse, Q, pages, q_len, table, k_len, heads, page, 2.0 ** -8, False, rows)
    within(got, lse, Q, pages, q_len, table, k_len, heads, page, 2.0 ** -11, False, ~rows)


@pytest.mark.parametrize("rows", ["few", "many"])
@pytest.mark.parametrize("by", [2.0 ** 100, 2.0 ** 116, 2.0 ** 121, 2.0 ** -60])
def test_values_at_the_ends_of_the_range(rows, by):
    """V's scales and offsets times a power of two: so is the result, to 2^127."""
    q_len, k_len, table, pages, Q, heads, page = setup(rows, 28)
    far = copied(pages)
    far.v_scale *= by
    got, lse = call(Q, far, q_len, table, k_len, heads)
    within((got.double() / by).float(), lse, Q, pages, q_len, table, k_len, heads, page, 2.0 ** -11, rows == "few")
