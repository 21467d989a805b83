"""What sp_cache_attention loses in the mean, against the formula in 64 bits: bf16 queries, values that average out over many keys.

The result is rounded to bf16: an error that is uniform within half a step, step / sqrt 12 in the mean, the steps those of the values that are expected.
Every other rounding of at most u relative to a value (2^-8 in bf16, 2^-11 in fp16) is u / sqrt 3 in the mean at most and adds up as squares: of
sum p v over keys with values of no common sign, the errors e of the terms leave sum p e v, whose size is e's share of the result's.  The mean of N squared
errors lies within 5 sqrt(3 / N) of what is expected (uniform within steps of different sizes: a fourth moment of four times the second's square), its
root within half of that."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api
from tests.test_gpu_paged_cache import gathered, gen, ints, offsets, table_for, values

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
FEW, MANY = ([1] * 12, [900 + 211 * i for i in range(12)]), ([300], [5000])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("four, lengths, roundings", [(True, FEW, [2.0 ** -11]), (False, FEW, [2.0 ** -16]),       # probabilities (times scales)
                                                      (True, MANY, [2.0 ** -11] * 3),                              # and opened values and keys
                                                      (False, MANY, [2.0 ** -8])])
def test_roundings_in_the_mean(four, lengths, roundings, dh):
    q_len, k_len = lengths
    heads, kv, page = 8, 2, 64
    table, n_pages = table_for(k_len, page, 51)
    g = gen(52)
    pages = api.KvPages.empty(n_pages, kv, page, dh, four)
    for x, s in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
        if four:
            n = (torch.randn(*x.shape[:3], dh, generator=g, device=DEV) * 2.7 + 7.5).round().clamp(0, 15).to(torch.uint8)
            x.copy_(n[..., 0::2] | n[..., 1::2] << 4)
            s[..., 0] = 0.37
            s[..., 1] = -7.5 * 0.37
        else:
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
    Q = torch.randn(sum(q_len), heads * dh, generator=g, device=DEV).to(BF)
    got, _ = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, max_keys=sum(k_len))
    (k64, _), (v64, _) = values(pages)
    cu, parts = offsets(q_len), []
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        K, V = gathered(k64, table, page, s, nk), gathered(v64, table, page, s, nk)
        z = torch.einsum("iagd,jad->agij", Q[cu[s]:cu[s + 1]].double().view(nq, kv, heads // kv, dh), K) * dh ** -0.5
        z = z.masked_fill(torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq, -math.inf)
        parts.append(torch.einsum("agij,jad->iagd", torch.softmax(z, 3), V).flatten(1))
    want = torch.cat(parts)
    step = 2.0 ** (want.abs().clamp_min(1e-30).log2().floor() - 7)
    expected = (step.square().mean() / 12 + sum(u * u for u in roundings) / 3 * want.square().mean()).sqrt()
    error = (got.double() - want).square().mean().sqrt()
    assert error <= expected * (1 + 2.5 * (3 / want.numel()) ** 0.5), (error / expected).item()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("lengths", [([1] * 40, [5 + 53 * i for i in range(40)]), ([4] * 10, [20 + 300 * i for i in range(10)])])
def test_lse_in_the_mean(lengths, four, dh):
    """Few rows.  A logit is a sum of some 16 partial sums in fp32 of terms <= T (by groups of 64 channels: scale <q, n> and offset sum q where 4 bits are
    opened so), each off by 2^-24 T / sqrt 3 in the mean at most; of a query's values 2^-22 of the row's largest are lost at most, 2^-22 / sqrt 3 in the mean,
    over the channels' numbers as squares.  lse averages the logits' errors, so it has no more than one logit's in the mean."""
    q_len, k_len = lengths
    heads, kv, page = 4, 2, 16
    table, n_pages = table_for(k_len, page, 53)
    g = gen(54)
    pages = api.KvPages.empty(n_pages, kv, page, dh, four)
    for x, s in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)):
        if four:
            x.copy_(torch.randint(0, 256, x.shape, generator=g, device=DEV))
            s[..., 0] = 0.1 + 0.3 * torch.rand(s.shape[:-1], generator=g, device=DEV)
            s[..., 1] = -7.5 * s[..., 0]
        else:
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
    Q = torch.randn(sum(q_len), heads * dh, generator=g, device=DEV)
    Q[:, ::16] *= 8.0                                             # strong channels: the others lie below a row's largest
    Q = Q.to(BF)
    _, lse = api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads, want_lse=True)
    (k64, k_size), _ = values(pages)
    cu, wrong, allowed = offsets(q_len), 0.0, 0.0
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        K, KS = gathered(k64, table, page, s, nk), gathered(k_size, table, page, s, nk)
        q = Q[cu[s]:cu[s + 1]].double().view(nq, kv, heads // kv, dh)
        z = torch.einsum("iagd,jad->agij", q, K) * dh ** -0.5
        hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq
        want = torch.logsumexp(z.masked_fill(hidden, -math.inf), 3)
        got = lse[cu[s]:cu[s + 1]].double().view(nq, kv, heads // kv).permute(1, 2, 0)
        wrong += (got - want).square().sum().item()
        if four:                                                   # |sum q| |offset| by groups, twice: the numbers' part is about as large
            off = (pages.k_scale[table[s, :-(-nk // page)].long()][..., 1].double().transpose(1, 2).flatten(0, 1)[:nk]).abs()
            T = 2 * torch.einsum("iagu,jau->agij", q.unflatten(3, (-1, 64)).sum(4).abs(), off)
            lost = torch.einsum("iag,ja->agij", q.abs().amax(3), KS.square().sum(2).sqrt()) * 2.0 ** -22
        else:
            T = torch.einsum("iagd,jad->agij", q.abs(), K.abs())
            lost = torch.zeros_like(T)
        one = ((16 * (T * 2.0 ** -24).square() + lost.square()) / 3 / dh).masked_fill(hidden, 0.0)
        allowed += one.amax(3).sum().item() + (2.0 ** -23 * want).square().sum().item()        # and lse's own last roundings
    assert wrong <= allowed, (wrong / allowed) ** 0.5
