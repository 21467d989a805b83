"""sp_cache_append, sp_cache_read and sp_cache_attention against their formulas in 64 bits.

Tolerances count roundings.  Turned values: cosine and sine within 2^-22, two products and a sum in fp32, 2^-21 of the pair's size in all, and half a
step of the type.  What 4 bits hold is compared exactly with the formula in 64 bits where no value lies within 2^-30 of a step from a border of two.
Attention: probabilities (in 4 bits their products with the scales) are rounded to bf16, half a step each: 2^-8 of sum p |scale n|, and the result
by half a step; in fp32 the logits are off by at most 2^-20 of the sum of their terms' magnitudes, which moves every p by as much."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def offsets(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def table_for(lens, page, seed=0, extra=2, width=0):
    """Scattered pages; entries behind a sequence's last page name no page."""
    need = [-(-n // page) for n in lens]
    total = sum(need) + extra
    order = torch.randperm(total, generator=gen(seed), device=DEV).int()
    table = torch.full((len(lens), max(max(need, default=0), 1) + width), 1 << 30, dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, total


def values(pages):
    """fp64 [n_pages, n_kv, page_len, d_head] that the pages stand for, and |scale n| + |zero| of them."""
    def of(x, s):
        if x.dtype != torch.uint8:
            return x.double(), x.double().abs()
        n = torch.stack((x & 15, x >> 4), -1).flatten(3).double().unflatten(3, (-1, 64))
        s = s.double()
        return (n * s[..., 0:1] + s[..., 1:2]).flatten(3), (n * s[..., 0:1].abs() + s[..., 1:2].abs()).flatten(3)
    return of(pages.k, pages.k_scale), of(pages.v, pages.v_scale)


def gathered(x, table, page, s, n):
    at = torch.arange(n, device=DEV)
    return x[table[s].long()[at // page], :, at % page]           # [n, kv, dh]


# ------------------------------------------------------------------------------------------------------------ append
def turn64(x, position, inv_freq, neighbours):
    n = inv_freq.numel()
    angle = position.double()[:, None, None] * inv_freq.double()
    c, s = angle.cos(), angle.sin()
    out = x.clone()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    u, v = a * c - b * s, b * c + a * s
    size = (a.abs() + b.abs())
    near = torch.zeros_like(x)
    if neighbours:
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = u, v
        near[..., 0:2 * n:2] = near[..., 1:2 * n:2] = size
    else:
        out[..., :n], out[..., n:2 * n] = u, v
        near[..., :n] = near[..., n:2 * n] = size
    return out, near


def four64(x):
    """x fp64 [T, kv, dh]: (held values, whether the number is certain)."""
    g = x.unflatten(2, (-1, 64))
    zero = g.amin(3, keepdim=True).float().bfloat16().double()
    scale = ((g.amax(3, keepdim=True) - zero) / 15).float().bfloat16().double()
    q = torch.where(scale > 0, (g - zero) / scale, torch.zeros_like(g))
    n = q.round().clamp(0, 15)
    sure = (q - q.floor() - 0.5).abs() > 2.0 ** -30
    sure |= q == q.floor() + 0.5                                  # (a tie is exact where the values are)
    return (n * scale + zero).flatten(2), sure.flatten(2)


def append_case(new, before, heads, kv, dh, page, dtype, four, turned, neighbours=False, seed=0, tail=0, in_place=False, positions=None,
                odd_layout=False):
    after = [a + b for a, b in zip(new, before)]
    table, n_pages = table_for(after, page, seed)
    N = sum(new) + tail
    pages = api.KvPages.empty(n_pages, kv, page, dh, four)
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0xff if t.dtype != torch.uint8 else 0xa5)
    before_k, before_v = pages.k.clone(), pages.v.clone()
    width = (heads + 2 * kv) * dh + (1 if odd_layout else 0)
    qkv = torch.randn(N + 1, width, generator=gen(seed + 1), device=DEV).to(dtype)[1 if odd_layout else 0:][:N]
    q, k, v = qkv[:, :heads * dh], qkv[:, heads * dh:(heads + kv) * dh], qkv[:, (heads + kv) * dh:(heads + 2 * kv) * dh]
    orig = qkv.clone()
    oq, ok, ov = (x.double().reshape(N, -1, dh) for x in (orig[:, :heads * dh], orig[:, heads * dh:(heads + kv) * dh],
                                                          orig[:, (heads + kv) * dh:(heads + 2 * kv) * dh]))
    inv_freq = 10000.0 ** (-2.0 * torch.arange(turned // 2, device=DEV).float() / max(turned, 1)) if turned else None
    status = api.new_status()
    cu = ints(offsets(new))
    q_out = q if in_place else torch.full((N, heads * dh), 9.0, dtype=dtype, device=DEV)
    k_out = torch.full((N, kv * dh), 9.0, dtype=dtype, device=DEV)
    got_q, got_k = api.sp_cache_append(pages, k, v, cu, table, ints(after), Q=q, inv_freq=inv_freq, neighbours=neighbours,
                                       positions=positions, q_out=q_out, k_out=k_out, status=status)
    assert status.tolist() == [0, 0, 0, 0]
    K, V = api.sp_cache_read(pages, cu, table, ints(after), N, F32, K=torch.full((N, kv * dh), 9.0, device=DEV),
                             V=torch.full((N, kv * dh), 9.0, device=DEV), status=status)
    assert status.tolist() == [0, 0, 0, 0]
    n = sum(new)
    place = torch.cat([torch.arange(b, b + a, device=DEV) for a, b in zip(new, before)]) if new else torch.zeros(0, device=DEV)
    where = place if positions is None else positions[:n]
    f = inv_freq if turned else torch.zeros(0, device=DEV)
    wq, near_q = turn64(oq[:n], where, f, neighbours)
    wk, near_k = turn64(ok[:n], where, f, neighbours)
    for got, want, near in ((got_q, wq, near_q), (got_k, wk, near_k)):
        want, near = want.flatten(1), near.flatten(1)
        assert ((got[:n].double() - want).abs() <= want.abs() * HALF[dtype] + near * 2.0 ** -21).all()
    assert (got_k[n:] == 9).all() and (K[n:] == 9).all() and (V[n:] == 9).all()
    assert torch.equal(got_q[n:], orig[n:, :heads * dh]) if in_place else (got_q[n:] == 9).all()
    if four:
        for got, want in ((K, four64(wk)), (V, four64(ov[:n]))):
            held, sure = (x.flatten(1) for x in want)
            far = (got[:n].double() - held).abs() > 2.0 ** -23 * held.abs().clamp_min(1e-3) + 1e-9
            assert not (far & sure).any() and sure.float().mean() > 0.999
    else:
        assert torch.equal(V[:n], ov[:n].flatten(1).float().bfloat16().float())
        want = wk.flatten(1)
        assert ((K[:n].double() - want).abs() <= want.abs() * HALF[BF] + near_k.flatten(1) * 2.0 ** -21).all()
    # nothing but the slots of the new tokens has changed
    touched = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
    for s, (a, b) in enumerate(zip(new, before)):
        at = torch.arange(b, b + a, device=DEV)
        touched[table[s].long()[at // page], at % page] = True
    for now, then in ((pages.k, before_k), (pages.v, before_v)):
        same = (now.view(torch.uint8) == then.view(torch.uint8)).all(3)
        assert (same | touched[:, None, :]).all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads, kv, dh", [(1, 1, 64), (12, 12, 64), (32, 8, 128), (5, 5, 128), (7, 1, 64)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append(four, dtype, heads, kv, dh, neighbours):
    append_case([1, 0, 17, 40, 1, 16], [0, 5, 15, 100000, 31, 0], heads, kv, dh, 16, dtype, four, dh, neighbours, tail=3)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("turned", [0, 16, 48, 96, 128])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append_turns_some_channels(four, turned, neighbours):
    append_case([9, 3], [77, 0], 4, 2, 128, 32, BF, four, turned, neighbours, seed=5)


@pytest.mark.parametrize("dh", [16, 48, 80, 96, 112])
def test_append_head_widths_of_16_bits(dh):
    append_case([5, 20], [3, 0], 6, 3, dh, 48, BF, False, dh // 32 * 16, seed=6)


@pytest.mark.parametrize("four", [False, True])
def test_append_layouts(four):
    append_case([5, 20], [3, 0], 4, 2, 64, 16, BF, four, 64, seed=7, odd_layout=True, tail=2)
    append_case([5, 20], [3, 0], 4, 2, 64, 16, F32, four, 64, seed=7, odd_layout=True)
    append_case([5, 20], [3, 0], 4, 2, 128, 16, BF, four, 96, seed=8, in_place=True, tail=2)
    append_case([5, 20], [3, 0], 4, 2, 128, 16, F32, four, 128, neighbours=True, seed=8, in_place=True)
    append_case([5, 20], [3, 0], 4, 2, 64, 16, BF, four, 64, seed=9, positions=ints(list(range(2000000, 2000025))))


def test_append_of_many_sequences():
    g = torch.Generator().manual_seed(3)
    new = torch.randint(0, 3, (1500,), generator=g).tolist()
    append_case(new, [7 * (i % 40) for i in range(1500)], 2, 1, 64, 16, BF, True, 64, seed=10)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_groups_of_odd_values(dtype):
    """Equal values, tiny and huge ranges, values on the border of two steps, NaN and infinities: what the numbers hold."""
    x = torch.zeros(12, 128, dtype=torch.float64, device=DEV)
    x[0] = 3.25
    x[1, :64] = torch.arange(64, device=DEV) / 64.0
    x[2] = torch.linspace(-1e-30, 1e-30, 128, device=DEV)
    x[3] = torch.linspace(-1e38, 1e38, 128, device=DEV)
    x[4] = (torch.arange(128, device=DEV) % 31) / 2.0 - 2         # steps of 1, half of the values on borders
    x[5] = 1e6 + torch.arange(128, device=DEV)
    x[6, 1] = 1e-40
    x[7] = torch.randn(128, device=DEV, generator=gen(1)).double() * 1e-38
    x[8] = -(torch.arange(128, device=DEV) % 31) / 2.0
    x = x.to(dtype)
    x[9, 70], x[10, 3], x[11, 5] = float("nan"), float("inf"), float("-inf")
    pages = api.KvPages.empty(1, 1, 16, 128, True)
    table, lens, cu = ints([[0]]), ints([12]), ints([0, 12])
    api.sp_cache_append(pages, x, x, cu, table, lens)
    K, V = api.sp_cache_read(pages, cu, table, lens, 12, F32)
    held, sure = four64(x[:9].double()[:, None].clone())
    for got in (K, V):
        far = (got[:9].double() - held.flatten(1)).abs() > 2.0 ** -23 * held.flatten(1).abs() + 1e-45
        assert not (far & sure.flatten(1)).any()
        assert got[9, 64:].isnan().all() and not got[9, :64].isnan().any()
        assert got[10, :64].isnan().all() and not got[10, 64:].isnan().any() and got[11, :64].isnan().all()


def test_turning_without_pages():
    q, k = torch.randn(30, 4 * 64, device=DEV), torch.randn(30, 2 * 64, device=DEV)
    f = 10000.0 ** (-2.0 * torch.arange(32, device=DEV).float() / 64)
    cu = ints([0, 10, 25])
    gq, gk = api.sp_cache_append(None, k, None, cu, None, None, Q=q, inv_freq=f, want_k=True, d_head=64)
    place = torch.cat((torch.arange(10), torch.arange(15))).to(DEV)
    for got, x in ((gq, q), (gk, k)):
        want, near = (t.flatten(1) for t in turn64(x[:25].double().view(25, -1, 64), place, f, False))
        assert ((got[:25].double() - want).abs() <= want.abs() * 2.0 ** -24 + near * 2.0 ** -21).all()


def test_places_without_a_page_are_reported_and_nothing_is_touched():
    pages = api.KvPages.empty(4, 1, 16, 64, True)
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        t.view(torch.uint8).fill_(7)
    k = torch.randn(6, 64, device=DEV)
    good = ints([[0], [1], [2]])
    for table, lens, seq in ((ints([[0], [4], [2]]), ints([2, 2, 2]), 1),           # an entry that names no page
                             (ints([[0], [1], [-1]]), ints([2, 2, 2]), 2),
                             (good, ints([18, 2, 2]), 0),                             # behind the table
                             (good, ints([2, 2, 1]), 2)):                             # fewer tokens than the call brings
        for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
            t.view(torch.uint8).fill_(7)
        status = api.new_status()
        api.sp_cache_append(pages, k, k, ints([0, 2, 4, 6]), table, lens, status=status)
        s = status.tolist()
        assert s[0] == 2 and s[1] == seq
        assert (pages.k[3].view(torch.uint8) == 7).all()
        status = api.new_status()
        K, V = api.sp_cache_read(pages, ints([0, 2, 4, 6]), table, lens, 6, F32, status=status)
        assert status.tolist()[:2] == [2, seq]
        bad = K.isnan().all(1)
        assert bad[2 * seq:2 * seq + 2].any() and not bad[[i for i in range(6) if i // 2 != seq]].any()
        assert torch.equal(bad, V.isnan().all(1))


# --------------------------------------------------------------------------------------------------------- attention
def filled(n_pages, kv, page, dh, four, seed):
    g = gen(seed)
    pages = api.KvPages.empty(n_pages, kv, page, dh, four)
    for x, s in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
        if four:
            x.copy_(torch.randint(0, 256, x.shape, generator=g, device=DEV))
            s[..., 0] = 0.1 + 0.3 * torch.rand(s.shape[:-1], generator=g, device=DEV)
            s[..., 1] = -7.5 * s[..., 0] + 0.3 * torch.randn(s.shape[:-1], generator=g, device=DEV)
        else:
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
    return pages


def check_attention(q_len, k_len, heads, kv, dh, page, dtype, four, causal=True, tail=0, seed=0, scale=None, pages=None, table=None, Q=None,
                    max_keys=0, **kw):
    if pages is None:
        table, n_pages = table_for(k_len, page, seed, width=1)
        pages = filled(n_pages, kv, page, dh, four, seed + 1)
    N = sum(q_len) + tail
    if Q is None:
        Q = torch.randn(N, heads * dh, generator=gen(seed + 2), device=DEV).to(dtype)
    out = torch.full((N, heads * dh), 5.0, dtype=dtype, device=DEV)
    lse = torch.full((N, heads), 5.0, device=DEV)
    status = api.new_status()
    api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, causal=causal, scale=scale, max_keys=max_keys, out=out,
                           lse=lse, status=status, **kw)
    assert status.tolist() == [0, 0, 0, 0]
    (k64, k_size), (v64, v_size) = values(pages)
    few = N * (heads // kv) <= 64 * len(q_len)
    g, cu = heads // kv, offsets(q_len)
    scale = dh ** -0.5 if scale is None else scale
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        if nq == 0:
            continue
        q = Q[cu[s]:cu[s + 1]].double().view(nq, kv, g, dh)
        K, V, KS, VS = (gathered(x, table, page, s, nk) for x in (k64, v64, k_size, v_size))
        z = torch.einsum("iagd,jad->agij", q, K) * scale
        hidden = torch.zeros(nq, nk, dtype=torch.bool, device=DEV)
        if causal:
            hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq
        z = z.masked_fill(hidden, -math.inf)
        want_lse = torch.logsumexp(z, 3) if nk else torch.full((kv, g, nq), -math.inf, device=DEV).double()
        p = torch.where(want_lse[..., None] == -math.inf, 0.0, (z - want_lse[..., None]).exp())
        want = torch.einsum("agij,jad->iagd", p, V)
        # logits: fp32 sums of products (opened values rounded to bf16 where there are many rows), and what that does to p
        z_size = torch.einsum("iagd,jad->agij", q.abs(), KS) * scale * 2.0 ** -19
        opened = dtype == BF and not few and four
        if opened:
            z_size = z_size + torch.einsum("iagd,jad->agij", q.abs(), K.abs()) * scale * 2.0 ** -8
        z_off = (p * z_size).sum(3) if nk else torch.zeros_like(want_lse)
        worst = z_size.amax(3) if nk else z_off
        off = torch.einsum("agij,jad->iagd", p * (z_size + z_off[..., None] + 2.0 ** -20), VS)
        if dtype == BF:
            off = off + 2.0 ** -8 * torch.einsum("agij,jad->iagd", p, VS) * (2 if opened else 1) + 2.0 ** -8 * want.abs()
        else:
            off = off + 2.0 ** -21 * torch.einsum("agij,jad->iagd", p, VS)
        got = out[cu[s]:cu[s + 1]].double().view(nq, kv, g, dh)
        assert ((got - want).abs() <= off + 1e-7).all(), (s, nq, nk, ((got - want).abs() - off).max().item())
        got = lse[cu[s]:cu[s + 1]].double().view(nq, kv, g).permute(1, 2, 0)
        none = want_lse == -math.inf
        assert torch.equal(got == -math.inf, none)
        assert ((got - want_lse).abs()[~none] <= (worst + 2.0 ** -20 * (1 + want_lse.abs()))[~none]).all()
    assert (out[sum(q_len):] == 5).all() and (lse[sum(q_len):] == 5).all()
    return out, lse


LENGTHS = [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 700, 1, 4097, 33]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads, kv, dh", [(12, 12, 64), (8, 2, 64), (32, 8, 128), (9, 1, 128), (16, 1, 64), (40, 2, 128)])
def test_single_tokens(four, dtype, heads, kv, dh):
    check_attention([1] * len(LENGTHS), LENGTHS, heads, kv, dh, 16, dtype, four, tail=2, seed=1)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads, kv, dh", [(4, 4, 64), (8, 1, 128), (14, 2, 128)])
def test_a_few_tokens_of_each(four, dtype, causal, heads, kv, dh):
    q = [1, 5, 3, 0, 8, 2, 7, 6, 1, 4]
    k = [1, 3, 17, 40, 300, 0, 7, 1029, 0, 2000]                 # queries without a key among them, more queries than keys
    check_attention(q, k, heads, kv, dh, 48, dtype, four, causal, tail=1, seed=2)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("max_keys", [0, 5000])
def test_many_tokens(four, dtype, causal, max_keys):
    check_attention([200, 1, 0, 333, 77], [1000, 5, 40, 333, 70], 8, 2, 128, 64, dtype, four, causal, tail=3, seed=3, max_keys=max_keys)
    check_attention([150], [2100], 4, 4, 64, 16, dtype, four, causal, seed=4, max_keys=max_keys)


@pytest.mark.parametrize("dh", [16, 48, 80, 96, 112])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_widths_of_16_bits(dh, dtype):
    check_attention([1] * 6, [1, 16, 300, 40, 900, 5], 6, 3, dh, 16, dtype, False, seed=5)
    check_attention([90, 100], [91, 400], 6, 3, dh, 16, dtype, False, seed=5)


@pytest.mark.parametrize("four", [False, True])
def test_parts_of_a_long_cache(four):
    """One long text, alone and among many short ones: the keys are cut into parts, and joined."""
    check_attention([1], [30011], 8, 2, 128, 64, BF, four, seed=6)
    check_attention([1, 4] + [1] * 40, [9000, 30011] + [3] * 40, 8, 2, 64, 32, BF, four, seed=7)
    check_attention([3], [20000], 4, 1, 128, 128, F32, four, seed=8)


def test_many_sequences():
    """More than one launch holds."""
    g = torch.Generator().manual_seed(5)
    n = 1100
    k = torch.randint(0, 60, (n,), generator=g).tolist()
    check_attention([i % 3 for i in range(n)], k, 4, 2, 64, 16, BF, True, seed=9)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_layouts(four, dtype):
    """Queries and results as column slices, an odd pitch, pages of several layers in one buffer, another scale."""
    q_len, k_len, heads, kv, dh, page = [1, 2, 1], [100, 37, 600], 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 11, width=3)
    table = torch.cat((table, torch.zeros(3, 2, dtype=torch.int32, device=DEV)), 1)[:, :-2]
    both = filled(n_pages, 3 * kv, page, dh, four, 12)
    cut = lambda x: None if x is None else x[:, kv:2 * kv]       # a layer's slice: contiguous within a page, pages apart
    pages = api.KvPages(*(cut(x) for x in (both.k, both.v, both.k_scale, both.v_scale)))
    wide = torch.randn(4, 3 * heads * dh + 1, generator=gen(13), device=DEV).to(dtype)
    Q = wide[:, 1:1 + heads * dh]
    a, la = check_attention(q_len, k_len, heads, kv, dh, page, dtype, four, pages=pages, table=table, Q=Q, scale=0.3)
    out = torch.full((4, heads * dh + 9), 2.0, dtype=dtype, device=DEV)
    got, _ = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, scale=0.3, out=out[:, 5:5 + heads * dh])
    assert torch.equal(got, a) and (out[:, :5] == 2).all() and (out[:, 5 + heads * dh:] == 2).all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_slots_that_a_query_does_not_see(four, dtype, rows):
    """NaN and infinities in slots behind the last token, and at keys that the mask hides from some queries, reach none that does not see them;
    seen, they make the channels of their group (4 bits) or their own (16) NaN or infinite."""
    q_len, k_len = ([6, 1], [50, 20]) if rows == "few" else ([120, 90], [300, 130])
    heads, kv, dh, page = 2, 1, 64, 16
    table, n_pages = table_for(k_len, page, 14)
    pages = filled(n_pages, kv, page, dh, four, 15)
    want, _ = check_attention(q_len, k_len, heads, kv, dh, page, dtype, four, pages=pages, table=table)
    bad = api.KvPages(*(None if x is None else x.clone() for x in (pages.k, pages.v, pages.k_scale, pages.v_scale)))
    hide = ([q_len[0] - 1] if rows == "few" else [100])[0]        # query `hide` of the first text sees the key, earlier ones do not
    key = k_len[0] - q_len[0] + hide
    spots = [(0, key)] + [(s, j) for s in (0, 1) for j in range(k_len[s], -(-k_len[s] // page) * page)]
    for s, j in spots:
        pg, slot = int(table[s, j // page]), j % page
        if four:
            bad.v_scale[pg, 0, slot, 0, 0] = float("nan")
            if j >= k_len[s]:
                bad.k_scale[pg, 0, slot] = float("inf")
        else:
            bad.v[pg, 0, slot, 3] = float("inf")
            if j >= k_len[s]:
                bad.k[pg, 0, slot] = float("nan")
                bad.v[pg, 0, slot] = float("nan")
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(2), device=DEV).to(dtype)
    got, lse = api.sp_cache_attention(Q, bad, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True)
    assert not lse.isnan().any()
    assert torch.equal(got[:hide], want[:hide]) and torch.equal(got[q_len[0]:], want[q_len[0]:])
    seen = got[hide:q_len[0]].view(-1, heads, dh)
    if four:
        assert seen.isnan().all()
    else:
        assert (~seen[..., 3].isfinite()).all() and seen[..., :3].isfinite().all() and seen[..., 4:].isfinite().all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("rows", ["few", "many"])
def test_pages_that_are_none(four, rows):
    q_len, k_len = ([2, 1, 3], [40, 300, 33]) if rows == "few" else ([90, 80, 100], [90, 300, 133])
    heads, kv, dh, page = 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 16)
    pages = filled(n_pages, kv, page, dh, four, 17)
    Q = torch.randn(sum(q_len), heads * dh, generator=gen(2), device=DEV).to(BF)
    want, _ = check_attention(q_len, k_len, heads, kv, dh, page, BF, four, pages=pages, table=table, Q=Q)
    cu = offsets(q_len)
    for entry in (-1, n_pages, 1 << 30):
        other = table.clone()
        other[1, 7] = entry
        status = api.new_status()
        got, lse = api.sp_cache_attention(Q, pages, ints(cu), other, ints(k_len), heads, want_lse=True, status=status)
        assert status.tolist()[:2] == [2, 1]
        ok = [i for i in range(sum(q_len)) if not cu[1] <= i < cu[2]]
        assert torch.equal(got[ok], want[ok]) and got[cu[1]:cu[2]].isnan().all() and lse[cu[1]:cu[2]].isnan().all()
    long = list(k_len)
    long[1] = table.shape[1] * page + 1                          # more tokens than the table has entries for
    status = api.new_status()
    got, _ = api.sp_cache_attention(Q, pages, ints(cu), table, ints(long), heads, status=status)
    assert status.tolist()[:2] == [2, 1] and torch.equal(got[ok], want[ok]) and got[cu[1]:cu[2]].isnan().all()
    if rows == "many":                                           # more keys than the caller said
        status = api.new_status()
        got, _ = api.sp_cache_attention(Q, pages, ints(cu), table, ints(k_len), heads, max_keys=k_len[0] + k_len[1], status=status)
        assert status.tolist()[:2] == [2, 2] and got[cu[2]:].isnan().all()
        # (the keys may be cut at other places than above: both calls are within 2^-8 sum p |v| + 2^-8 |o| of the formula, sum p = 1, |o| <= |v|)
        top = values(pages)[1][0].abs().max().item()
        assert (got[:cu[2]].double() - want[:cu[2]].double()).abs().max().item() <= 4 * 2.0 ** -8 * top


@pytest.mark.parametrize("four", [False, True])
def test_peaked_rows_and_large_logits(four):
    """Logits far apart: references rise many times on the way."""
    heads, kv, dh, page = 4, 1, 64, 16
    k_len = [2000]
    table, n_pages = table_for(k_len, page, 18)
    pages = filled(n_pages, kv, page, dh, four, 19)
    order = torch.arange(2000, device=DEV)
    grow = (pages.k_scale if four else pages.k)
    for j in range(0, 2000, 50):                                 # keys grow along the text
        pg, slot = int(table[0, j // page]), j % page
        grow[pg, 0, slot] *= 1 + j / 100
    assert order.numel() == 2000
    check_attention([1], k_len, heads, kv, dh, page, BF, four, pages=pages, table=table, seed=20)
    check_attention([1], k_len, heads, kv, dh, page, F32, four, pages=pages, table=table, seed=20)


@pytest.mark.parametrize("four", [False, True])
def test_captured_and_on_other_streams(four):
    """Two captured graphs with a workspace each replay side by side; lengths and tables are read when they run."""
    heads, kv, dh, page = 8, 2, 128, 16
    k_len = [3000, 700]
    table, n_pages = table_for(k_len, page, 21)
    pages = filled(n_pages, kv, page, dh, four, 22)
    lens, cu = ints(k_len), ints([0, 1, 2])
    Q = torch.randn(2, heads * dh, generator=gen(23), device=DEV).to(BF)
    want = api.sp_cache_attention(Q, pages, cu, table, lens, heads)[0].clone()
    shorter = api.sp_cache_attention(Q, pages, cu, table, ints([1111, 64]), heads)[0].clone()
    need = api.lib().sp_cache_attention_bytes(2, 2, heads, kv, dh, api.SP_BF16, table.shape[1], page, 0)
    graphs = []
    for _ in range(2):
        ws, out, s = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty_like(Q), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            api.sp_cache_attention(Q, pages, cu, table, lens, heads, out=out, ws=ws)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                api.sp_cache_attention(Q, pages, cu, table, lens, heads, out=out, ws=ws)
        graphs.append((g, s, out))
    torch.cuda.synchronize()
    for expect, now in ((want, k_len), (shorter, [1111, 64]), (want, k_len)):
        lens.copy_(ints(now))
        for _, _, out in graphs:
            out.zero_()
        torch.cuda.synchronize()
        for g, s, _ in graphs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, _, out in graphs:
            assert torch.equal(out, expect)


@pytest.mark.parametrize("q_len, k_len", [([1], [16000]), ([3, 1], [5000, 9000]), ([300], [8000])])
def test_four_bits_lose_no_more_than_their_roundings(q_len, k_len):
    """bf16: the result is rounded (half a step, 2^-8 of the value at most and uniform below: 2^-8 / sqrt 3 in the mean), the probabilities are as
    much, and with many rows the opened values; these add up as squares over thousands of keys whose values average out."""
    heads, kv, dh, page = 4, 2, 128, 64
    table, n_pages = table_for(k_len, page, 31)
    g = gen(32)
    pages = api.KvPages.empty(n_pages, kv, page, dh, True)
    for x, s in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
        n = (torch.randn(*x.shape[:3], dh, generator=g, device=DEV) * 2.7 + 7.5).round().clamp(0, 15).to(torch.uint8)
        x.copy_(n[..., 0::2] | n[..., 1::2] << 4)
        s[..., 0] = 0.37
        s[..., 1] = -7.5 * 0.37
    Q = (2 * torch.randn(sum(q_len), heads * dh, generator=g, device=DEV)).to(BF)
    got, _ = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, max_keys=sum(k_len))
    (k64, _), (v64, _) = values(pages)
    want, cu = torch.zeros(sum(q_len), heads, dh, dtype=torch.float64, device=DEV), offsets(q_len)
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        K, V = gathered(k64, table, page, s, nk), gathered(v64, table, page, s, nk)
        z = torch.einsum("iagd,jad->agij", Q[cu[s]:cu[s + 1]].double().view(nq, kv, heads // kv, dh), K) * dh ** -0.5
        z = z.masked_fill(torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq, -math.inf)
        want[cu[s]:cu[s + 1]] = torch.einsum("agij,jad->iagd", torch.softmax(z, 3), V).flatten(1, 2)
    roundings = 2 if sum(q_len) * (heads // kv) <= 64 * len(q_len) else 3
    assert (got.double() - want.flatten(1)).norm() <= (roundings / 3) ** 0.5 * 2.0 ** -8 * want.norm()


@pytest.mark.parametrize("q_len, k_len", [([1], [900]), ([3, 1], [40, 700]), ([200], [500])])
def test_scales_of_very_different_sizes(q_len, k_len):
    """Scales of V that grow a thousandfold on the way, and leftovers of any size in slots that hold no token of the text."""
    heads, kv, dh, page = 4, 2, 64, 16
    table, n_pages = table_for(k_len, page, 41)
    pages = filled(n_pages, kv, page, dh, True, 42)
    for s, n in enumerate(k_len):
        for j in range(n):
            pg, slot = int(table[s, j // page]), j % page
            if j % 37 == 0:
                pages.v_scale[pg, :, slot] *= 2.0 ** (10 * j / n) if j % 2 else 2.0 ** -9
    want, want_lse = check_attention(q_len, k_len, heads, kv, dh, page, BF, True, pages=pages, table=table, seed=43)
    check_attention(q_len, k_len, heads, kv, dh, page, F32, True, pages=pages, table=table, seed=43)
    left = api.KvPages(*(x.clone() for x in (pages.k, pages.v, pages.k_scale, pages.v_scale)))
    for s, n in enumerate(k_len):
        for j in range(n, -(-n // page) * page):
            pg, slot = int(table[s, j // page]), j % page
            for x in (left.k_scale, left.v_scale):
                x[pg, :, slot] = 3e38 if j % 2 else -2e38
    for dtype in (BF, F32):
        Q = torch.randn(sum(q_len), heads * dh, generator=gen(45), device=DEV).to(dtype)
        a = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True)
        b = api.sp_cache_attention(Q, left, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("q_len, k_len, heads, kv", [([16], [3000], 32, 8), ([17], [3000], 32, 8), ([12], [700], 128, 32), ([13], [700], 128, 32),
                                                      ([20, 20], [900, 30], 32, 8), ([22, 19], [900, 300], 32, 8), ([128], [2000], 2, 2)])
def test_on_both_sides_of_few_rows(q_len, k_len, heads, kv, four):
    check_attention(q_len, k_len, heads, kv, 64, 16, BF, four, seed=41, max_keys=sum(k_len))


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("max_keys", [0, 5003, 60000])
def test_a_chunk_of_one_text_whose_keys_are_cut(max_keys, causal, four):
    """Parts by what the caller says, right, too large or not at all: the text's length comes from the device."""
    check_attention([130], [5003], 8, 2, 128, 64, BF, four, causal, tail=2, seed=42, max_keys=max_keys)
    check_attention([3, 300], [60, 4000], 8, 2, 64, 16, BF, four, causal, seed=43, max_keys=max_keys)
