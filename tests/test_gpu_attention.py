"""sp_attention against the definition in 64 bits.

Tolerances, per entry of O: the probabilities are rounded to the storage type before the second product (bf16: at most half a
step, 2^-8 of each; fp32 mode: 2^-24), which moves O by at most that times A = sum_j p_j |V_j|; the result is rounded once
(the same share of |O|); a logit is a sum of d_head products in fp32, off by at most (d_head + 4) 2^-23 sum |q k| scale =: e
(one step per addition covers chopped as well as rounded additions), which moves every p by a factor within 1 +- 2 e;
exponentials, sums of n terms and the rescalings add (n + 32) 2^-23."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def offsets(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def cu(lengths):
    return torch.tensor(offsets(lengths), dtype=torch.int32, device=DEV)


def reference(Q, K, V, q_len, k_len, heads, kv, causal, scale):
    """O, lse, and the bounds on their errors, in 64 bits; rows of no sequence are NaN."""
    dh = Q.shape[1] // heads
    half = HALF[Q.dtype]
    O = torch.full((Q.shape[0], heads * dh), math.nan, dtype=torch.float64, device=DEV)
    lse = torch.full((Q.shape[0], heads), math.nan, dtype=torch.float64, device=DEV)
    tol_o, tol_l = torch.zeros_like(O), torch.zeros_like(lse)
    oq, ok = offsets(q_len), offsets(k_len)
    for s, (nq, nk) in enumerate(zip(q_len, k_len)):
        rq, rk = slice(oq[s], oq[s] + nq), slice(ok[s], ok[s] + nk)
        for h in range(heads):
            j = h // (heads // kv)
            q, k = Q[rq, h * dh:(h + 1) * dh].double(), K[rk, j * dh:(j + 1) * dh].double()
            v = V[rk, j * dh:(j + 1) * dh].double()
            z = q @ k.T * scale
            e = (q.abs() @ k.abs().T) * scale * (dh + 4) * 2.0 ** -23
            hidden = torch.zeros(nq, nk, dtype=torch.bool, device=DEV)
            if causal:
                hidden = torch.ones(nq, nk, dtype=torch.bool, device=DEV).triu(nk - nq + 1)
            z = z.masked_fill(hidden, -math.inf)
            e = e.masked_fill(hidden, 0).amax(1, keepdim=True) if nk else torch.zeros(nq, 1, dtype=torch.float64, device=DEV)
            m = z.amax(1, keepdim=True) if nk else torch.full((nq, 1), -math.inf, dtype=torch.float64, device=DEV)
            m = torch.where(m == -math.inf, 0.0, m)
            p = (z - m).exp()
            l = p.sum(1, keepdim=True)
            p = p / l.clamp_min(1e-300)
            v0 = torch.nan_to_num(v)
            cols = slice(h * dh, (h + 1) * dh)
            O[rq, cols] = p @ v0
            lse[rq, h] = (m + l.log()).squeeze(1)
            fixed = 2 * e + (nk + 32) * 2.0 ** -23
            tol_o[rq, cols] = (half + fixed) * (p @ v0.abs()) + half * O[rq, cols].abs()
            tol_l[rq, h] = (fixed + 2.0 ** -22 * (m.abs() + 1)).squeeze(1)
    return O, lse, tol_o, tol_l


def check(Q, K, V, q_len, k_len, heads, kv, causal=True, scale=None, **kw):
    dh = Q.shape[1] // heads
    o, l = api.sp_attention(Q, K, V, cu(q_len), cu(k_len), heads, kv, causal=causal, scale=scale, want_lse=True, **kw)
    O, L, tol_o, tol_l = reference(Q, K, V, q_len, k_len, heads, kv, causal, dh ** -0.5 if scale is None else scale)
    n = sum(q_len)
    err = (o[:n].double() - O[:n]).abs()
    assert torch.isfinite(o[:n]).all()
    assert (err <= tol_o[:n]).all(), float((err / tol_o[:n].clamp_min(1e-30)).max())
    none = L[:n] == -math.inf
    assert torch.equal(l[:n] == -math.inf, none)
    assert ((l[:n].double() - L[:n]).abs() <= tol_l[:n])[~none].all()
    assert (o[:n].unflatten(1, (heads, dh))[none] == 0).all()
    return o, l


def inputs(nq, nk, heads, kv, dh, dtype, seed=0, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda n, c: torch.randn(n, c, generator=g, device=DEV)
    return (spread * r(nq, heads * dh)).to(dtype), r(nk, kv * dh).to(dtype), r(nk, kv * dh).to(dtype)


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [8, 40, 64, 72, 128])
def test_head_sizes_and_ragged_sequences(dtype, causal, dh):
    lengths = [1, 63, 64, 65, 128, 0, 129, 255, 300]
    Q, K, V = inputs(sum(lengths), sum(lengths), 4, 2, dh, dtype)
    check(Q, K, V, lengths, lengths, 4, 2, causal)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (5, 5), (7, 1), (12, 4), (16, 2), (130, 2), (70, 1), (256, 2)])
def test_grouped_heads(dtype, heads, kv):
    q, k = [37, 1, 130], [37, 400, 260]
    Q, K, V = inputs(sum(q), sum(k), heads, kv, 64, dtype, seed=heads)
    check(Q, K, V, q, k, heads, kv)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_seq", [1, 3, 40, 200])
def test_single_tokens_after_caches_of_any_length(dtype, n_seq):
    k = [(i * 977) % 5000 + (i % 3 > 0) for i in range(n_seq)]
    k[0] = 5000
    Q, K, V = inputs(n_seq, sum(k), 8, 2, 128, dtype, seed=n_seq)
    check(Q, K, V, [1] * n_seq, k, 8, 2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_next_tokens_of_a_text_see_what_came_before(dtype):
    q, k = [5, 200, 1, 64], [1200, 1000, 1, 64]
    Q, K, V = inputs(sum(q), sum(k), 6, 3, 64, dtype)
    check(Q, K, V, q, k, 6, 3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_queries_without_a_visible_key(dtype):
    """More queries than keys: the first ones see nothing; a sequence without keys; one without queries."""
    q, k = [100, 3, 0, 300, 70], [60, 0, 50, 1, 70]
    Q, K, V = inputs(sum(q), sum(k), 4, 4, 64, dtype)
    check(Q, K, V, q, k, 4, 4)
    check(Q, K, V, q, k, 4, 4, causal=False)
    check(Q[:3], K[:0], V[:0], [3], [0], 4, 4)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_outside_the_sequences(dtype):
    """They are left as they were, and what stands in K and V there reaches nobody; neither do the sequences each other."""
    lengths = [70, 200]
    n, tail = sum(lengths), 77
    Q, K, V = inputs(n + tail, n + tail, 4, 2, 64, dtype)
    for t in (K, V, Q):
        t[n:] = math.nan
        t[n + 1::2] = math.inf
    out = torch.full((n + tail, 256), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((n + tail, 4), 7.0, device=DEV)
    check(Q, K, V, lengths, lengths, 4, 2, out=out, lse=lse)
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    V2, K2 = V.clone(), K.clone()
    V2[70:n] = math.nan
    K2[70:n] = math.nan
    o1, _ = api.sp_attention(Q, K, V, cu(lengths), cu(lengths), 4, 2)
    o2, _ = api.sp_attention(Q, K2, V2, cu(lengths), cu(lengths), 4, 2)
    assert torch.equal(o1[:70], o2[:70])
    # offsets that start behind the first row
    c = torch.tensor([70, n], dtype=torch.int32, device=DEV)
    out.fill_(7.0)
    api.sp_attention(Q, K, V, c, c, 4, 2, out=out)
    assert (out[:70] == 7).all() and (out[n:] == 7).all()
    alone, _ = api.sp_attention(Q[70:n], K[70:n], V[70:n], cu([200]), cu([200]), 4, 2)
    assert torch.equal(out[70:n], alone)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [3, 64, 127, 130, 299])
def test_bad_values_behind_the_causal_mask(dtype, at):
    n = 300
    Q, K, V = inputs(n, n, 4, 2, 64, dtype)
    good, _ = api.sp_attention(Q, K, V, cu([n]), cu([n]), 4, 2)
    for bad in (math.nan, math.inf, -math.inf):
        V2, K2 = V.clone(), K.clone()
        V2[at, 5] = bad
        o, _ = api.sp_attention(Q, K, V2, cu([n]), cu([n]), 4, 2)
        assert torch.equal(o[:at], good[:at])
        assert not torch.isfinite(o[at:, 5]).any()               # column 5 of the first key head: query heads 0 and 1
        assert torch.equal(o[at:, 6:64], good[at:, 6:64]) and torch.equal(o[:, 128:], good[:, 128:])
        K2[at] = bad
        o, _ = api.sp_attention(Q, K2, V, cu([n]), cu([n]), 4, 2)
        assert torch.equal(o[:at], good[:at])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread", [30.0, 300.0])
def test_peaked_rows(dtype, spread):
    """Logits of some hundreds: the running maximum rises by much, and most probabilities vanish."""
    q = [333]
    Q, K, V = inputs(333, 333, 2, 1, 64, dtype, spread=spread)
    # keys that grow along the sequence, so that the maximum rises in tile after tile
    K *= torch.linspace(0.05, 1.0, 333, device=DEV)[:, None].to(dtype)
    check(Q, K, V, q, q, 2, 1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_slices_of_one_matrix_odd_pitches_and_starts(dtype):
    heads, kv, dh, n = 4, 2, 64, 150
    qkv = torch.randn(n, (heads + 2 * kv) * dh, device=DEV).to(dtype)
    Q, K, V = qkv[:, :256], qkv[:, 256:384], qkv[:, 384:]
    out = torch.zeros(n, 300, dtype=dtype, device=DEV)[:, 11:267]       # rows that start anywhere
    o, _ = check(Q, K, V, [100, 50], [100, 50], heads, kv, out=out)
    same, _ = api.sp_attention(Q.contiguous(), K.contiguous(), V.contiguous(), cu([100, 50]), cu([100, 50]), heads, kv)
    assert torch.equal(o, same)
    odd = torch.randn(n, 515, device=DEV).to(dtype)                     # neither 16-byte pitch nor start
    check(odd[:, 1:257], odd[:, 257:385], odd[:, 386:514], [100, 50], [100, 50], heads, kv)
    check(odd[:, 1:29], odd[:, 257:264], odd[:, 386:393], [100, 50], [100, 50], 4, 1)     # heads of 7


@pytest.mark.parametrize("dtype", DTYPES)
def test_scale_and_repeatability(dtype):
    q = [400, 30]
    Q, K, V = inputs(430, 430, 8, 8, 128, dtype)
    a, la = check(Q, K, V, q, q, 8, 8, scale=0.31)
    b, lb = api.sp_attention(Q, K, V, cu(q), cu(q), 8, 8, scale=0.31, want_lse=True)
    assert torch.equal(a, b) and torch.equal(la, lb)
    c, none = api.sp_attention(Q, K, V, cu(q), cu(q), 8, 8, scale=0.31)
    assert none is None and torch.equal(a, c)


def test_offsets_beyond_32_bits():
    """A cache of which the last rows lie more than 2^32 bytes (and 2^31 elements) behind the first."""
    n, heads, dh = (1 << 31) // 1024 + 300, 8, 128
    K = torch.zeros(n, heads * dh, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros(n, heads * dh, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    K[-300:] = torch.randn(300, heads * dh, generator=g, device=DEV).bfloat16()
    V[-300:] = torch.randn(300, heads * dh, generator=g, device=DEV).bfloat16()
    Q = torch.randn(2, heads * dh, generator=g, device=DEV).bfloat16()
    c = torch.tensor([0, n - 300, n], dtype=torch.int32, device=DEV)
    o, _ = api.sp_attention(Q, K, V, cu([1, 1]), c, heads)
    O, _, tol, _ = reference(Q[1:], K[-300:], V[-300:], [1], [300], heads, heads, True, dh ** -0.5)
    assert ((o[1:].double() - O).abs() <= tol).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_another_stream_and_a_captured_call(dtype):
    q, k = [1, 1, 50], [700, 4000, 1300]                 # cut along the keys: two launches and a workspace
    Q, K, V = inputs(52, 6000, 8, 2, 64, dtype)
    want, want_lse = check(Q, K, V, q, k, 8, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, l = api.sp_attention(Q, K, V, cu(q), cu(k), 8, 2, want_lse=True)
    side.synchronize()
    assert torch.equal(o, want) and torch.equal(l, want_lse)
    out, lse, cq, ck = torch.zeros_like(want), torch.zeros_like(want_lse), cu(q), cu(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.sp_attention(Q, K, V, cq, ck, 8, 2, out=out, lse=lse)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # a replay reads the offsets and values of its time
    Q.mul_(0.5)
    ck.copy_(cu([600, 4100, 1300]))
    graph.replay()
    O, _, tol, _ = reference(Q, K, V, q, [600, 4100, 1300], 8, 2, True, 64 ** -0.5)
    assert ((out.double() - O).abs() <= tol).all()


def test_a_batch_gives_what_its_sequences_give_alone():
    """Both within the bound of the definition, so within twice that of each other."""
    q, k = [300, 40, 513, 7], [300, 90, 513, 7]
    Q, K, V = inputs(sum(q), sum(k), 32, 8, 128, torch.bfloat16)
    o, _ = check(Q, K, V, q, k, 32, 8)
    oq, ok = offsets(q), offsets(k)
    for s in range(4):
        rq, rk = slice(oq[s], oq[s + 1]), slice(ok[s], ok[s + 1])
        a, _ = check(Q[rq], K[rk], V[rk], [q[s]], [k[s]], 32, 8)
        tol = reference(Q[rq], K[rk], V[rk], [q[s]], [k[s]], 32, 8, True, 128 ** -0.5)[2]
        assert ((a.double() - o[rq].double()).abs() <= 2 * tol).all()


def test_bad_values_behind_the_mask_with_keyless_sequences_between():
    """Work without keys does not wait for the tensor core: what is known of one tile's values must not be lost to a later one's.  Rounds of
    as many equal sequences as there are SMs: infinite values, 31 rounds without keys, infinite values."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    nq, nk = 40, 30
    k = [nk] * sms + [0] * (31 * sms) + [nk] * sms
    q = [nq] * len(k)
    Q, K, V = inputs(sum(q), sum(k), 1, 1, 64, torch.bfloat16)
    good, _ = api.sp_attention(Q, K, V, cu(q), cu(k), 1)
    V2 = V.clone()
    V2.view(-1, nk, 64)[:, 20, 5] = math.inf                        # seen by queries 30 and later
    o, _ = api.sp_attention(Q, K, V2, cu(q), cu(k), 1)
    rows = torch.cat([o[:sms * nq], o[-sms * nq:]]).view(-1, nq, 64)
    want = torch.cat([good[:sms * nq], good[-sms * nq:]]).view(-1, nq, 64).clone()
    want[:, 30:, 5] = math.inf
    assert torch.equal(rows, want)
    assert (o[sms * nq:-sms * nq] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dh", [64, 72])
@pytest.mark.parametrize("heads,kv", [(2, 2), (3, 1), (8, 1), (10, 1), (16, 1)])
def test_few_rows_of_each_group(dtype, dh, heads, kv):
    """Single tokens with 1 to 16 rows per key head; a query matrix that starts anywhere; non-finite values in rows of no sequence."""
    q, k = [1, 1, 1, 2, 0, 1], [1, 64, 700, 1601, 30, 0]
    if heads // kv > 8:
        q[3] = 1
    n, m = sum(q), sum(k)
    Q, K, V = inputs(n, m + 70, heads, kv, dh, dtype, seed=heads)
    K[m:], V[m:] = math.nan, math.inf
    check(Q, K, V, q, k, heads, kv)
    check(Q, K, V, q, k, heads, kv, causal=False)
    buf = torch.zeros(n, heads * dh + 9, dtype=dtype, device=DEV)
    buf[:, 3:3 + heads * dh] = Q
    check(buf[:, 3:3 + heads * dh], K, V, q, k, heads, kv)


def test_wide_heads_of_long_fp32_sequences():
    q = [2401, 2300, 2500, 2399]
    Q, K, V = inputs(sum(q), sum(q), 8, 8, 72, torch.float32)
    check(Q, K, V, q, q, 8, 8)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_single_row_has_no_pitch(dtype):
    """One query and one key: the leading dimensions are not used, whatever they are."""
    Q, K, V = inputs(1, 1, 2, 2, 64, dtype)
    O = torch.zeros(1, 128, dtype=dtype, device=DEV)
    c = cu([1])
    code = api._DTYPES[dtype]
    args = api.SpAttentionArgs(*(api.SpMat(t.data_ptr(), code, 0, 1, 128, ld) for t, ld in ((Q, 0), (K, 5), (V, 3), (O, 0))),
                               c.data_ptr(), c.data_ptr(), None, 1, 2, 2, 1, 0.125)
    assert api.lib().sp_attention(api.C.byref(args), None, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(O, V)                                        # the one probability is 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
def test_many_sequences_of_any_length(dtype, causal, dh):
    """More than 32 of them, of very different lengths, some empty: every row is written once, by its own keys."""
    q = [(i * 37) % 151 for i in range(75)]
    k = [(i * 53) % 211 for i in range(75)]
    q[40], k[40], q[64], k[64] = 700, 900, 0, 300
    Q, K, V = inputs(sum(q), sum(k), 4, 2, dh, dtype)
    check(Q, K, V, q, k, 4, 2, causal)


def test_many_tiles_of_many_heads():
    """Several rounds of work for every SM, tiles of one and of two halves in turn."""
    q = [65, 700, 1, 129, 33, 1025, 64, 300, 97, 16] * 2
    Q, K, V = inputs(sum(q), sum(q), 24, 12, 128, torch.bfloat16)
    check(Q, K, V, q, q, 24, 12)
    Q, K, V = inputs(sum(q), sum(q), 24, 12, 64, torch.bfloat16)
    check(Q, K, V, q, q, 24, 12)


@pytest.mark.parametrize("dtype", DTYPES)
def test_calls_side_by_side_on_two_streams(dtype):
    """Each has a workspace of its own: the bits of a call by itself."""
    q, k = [1, 1, 1], [5000, 3000, 700]
    sets = [inputs(3, 8700, 8, 2, 64, dtype, seed=i) for i in range(2)]
    cq, ck = cu(q), cu(k)
    want = [api.sp_attention(*t, cq, ck, 8, 2)[0] for t in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for stream, t in zip(streams, sets):
            with torch.cuda.stream(stream):
                got.append(api.sp_attention(*t, cq, ck, 8, 2)[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
