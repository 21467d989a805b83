"""Values and batches at the edges of the operators: rows of few numbers, logits far from zero, logits beyond fp32, sequences of very
different lengths in one call."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api, pipeline
from tests import test_gpu_attention as att

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def best(x, n):
    """Indices of the n best logits of every row: falling, the lower index first, NaN behind all."""
    y = torch.where(torch.isnan(x), -math.inf, x.double())
    order = torch.sort(y, dim=1, descending=True, stable=True).indices
    nan = torch.isnan(x).gather(1, order)
    return order.gather(1, torch.sort(nan.int(), dim=1, stable=True).indices)[:, :n]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_alts", [1, 8, 32])
@pytest.mark.parametrize("V", [40, 600, 4097, 9001, 70001])
def test_alternatives_of_rows_of_few_numbers(dtype, V, n_alts):
    """Rows of NaN but for some: every place is written, NaN behind all numbers and in the order of their indices."""
    x = torch.full((9, V), math.nan, dtype=dtype, device=DEV)
    x[1, V // 2] = 3.0
    x[2, [V - 1, 5, V // 3]] = torch.tensor([1.0, 1.0, -2.0], dtype=dtype, device=DEV)
    x[3, 7:20] = -math.inf
    x[4, ::2] = 0.5
    x[5, 1:] = -math.inf
    x[6] = -math.inf
    x[6, V // 4] = math.nan
    x[7] = torch.randn(V, device=DEV).to(dtype)
    x[7, ::3] = math.nan
    x[8, 11] = math.inf
    ids = torch.full((9, n_alts), -7, dtype=torch.int32, device=DEV)
    alt = torch.full((9, n_alts), 7.0, device=DEV)
    m = api.mat(x)
    assert api.lib().sp_token_logprobs(api.C.byref(m), None, 1.0, n_alts, None, None, None, ids.data_ptr(), alt.data_ptr(), None,
                                       torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(ids.long(), best(x, n_alts))
    assert torch.isnan(alt).all()                                  # a row with a NaN has no log probabilities


def far_rows(V, dtype, seed=0):
    """Rows whose lse is far from zero, beside ordinary ones."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = torch.randn(9, V, generator=g, device=DEV)
    low = torch.finfo(dtype).min
    x = n.to(dtype)
    x[1] = low                                                     # a mask that leaves nothing
    x[2] = low
    x[2, V // 2:] = -math.inf
    x[3] = (300 * n[3] + 5e4).to(dtype)
    x[4] = (n[4] - 3000).to(dtype)
    x[5] = (1e30 * n[5]).to(dtype)
    x[6] = torch.finfo(dtype).max
    x[7] = -math.inf                                               # nothing at all
    x[8] = (-1e37 * n[8].abs()).to(dtype)
    x[8, ::2] = low
    return x, torch.randint(0, (V + 1) // 2, (9,), generator=g, device=DEV)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1.0, 0.5, 1.6])
@pytest.mark.parametrize("V", [1, 7, 1000, 4099, 50257])
@pytest.mark.parametrize("in_place", [False, True])
def test_gradient_of_rows_far_from_zero(dtype, scale, V, in_place):
    """fp32 does not hold the lse of such rows as exactly as p = e^(z - lse) needs it (in a row of nothing but the type's lowest value, log V
    is lost beside it, and with a scale above 1 it overflows).

    Tolerance: with the row's largest logit r, z - z_r is formed from a difference and a scale, each rounded once (with log2(e) once more), and
    the product: 4 half steps of 2^-24 of |z - z_r|; the log of the sum adds one per value of a thread (V / 256) and 16 for the joins;
    the exponential 2^-21.  That is e, the error of log p; p is off by a factor within 1 +- 1.1 e, p log p by p (e + 1.1 e |log p|), and
    the result is rounded once."""
    x, t = far_rows(V, dtype)
    r = api.sp_token_logprobs(x, t, scale=scale)
    g = torch.Generator(device=DEV).manual_seed(1)
    gl, gh = torch.randn(9, generator=g, device=DEV), torch.randn(9, generator=g, device=DEV)
    z = x.double() * scale
    empty = (x == -math.inf).all(1)
    zr = torch.where(empty, 0.0, z.amax(1))[:, None]
    lp = torch.where(empty[:, None], -math.inf, torch.log_softmax(z, 1))
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, 0.0)
    one = torch.zeros_like(p)
    one[torch.arange(9, device=DEV), t] = 1.0
    gap = torch.where(p > 0, (z - zr).abs(), 0.0)
    e = 2.0 ** -22 * gap + 2.0 ** -24 * (V / 256 + 16) + 2.0 ** -21
    e = torch.where(r.lse.abs()[:, None] < 1024, e + 2.0 ** -24 * 6 * torch.where(p > 0, z.abs() + lp.abs(), 0.0), e)     # from the lse as given
    for ent in (False, True):
        buf = x.clone()
        d = api.sp_token_logprobs_grad(buf, t, r.lse, gl, entropy=r.entropy if ent else None, g_entropy=gh if ent else None, scale=scale,
                                       out=buf if in_place else None)
        a, h = gl.double()[:, None], (gh.double()[:, None] if ent else torch.zeros(9, 1, dtype=torch.float64, device=DEV))
        H = r.entropy.double()[:, None]
        want = scale * (a * (one - p) - h * (plp + p * H))
        want[empty] = 0.0
        tol = scale * (1.1 * e * p * a.abs() + h.abs() * (p * e + 1.1 * e * (plp.abs() + p * H)))
        tol = tol + 2.0 ** -22 * scale * (a.abs() * (one + p) + h.abs() * (plp.abs() + p * H)) + HALF[dtype] * want.abs() + 1e-37
        # a p below 2^-126 becomes 0: p |log p| rises with p there, so at most 2^-126 times 126 log 2 < 88 is lost (4e-37 where it was first seen)
        tol = tol + 2.0 ** -126 * scale * (a.abs() + h.abs() * (88 + H))
        err = (d.double() - want).abs()
        assert torch.isfinite(d).all() and (err <= tol).all(), (float((err / tol).max()), (err / tol).argmax().item() // V)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_of_far_rows_with_pitches_and_nan(dtype):
    V = 1001
    x, t = far_rows(V, dtype)
    r = api.sp_token_logprobs(x, t)
    gl = torch.ones(9, device=DEV)
    want = api.sp_token_logprobs_grad(x, t, r.lse, gl)
    src = torch.full((9, 1200), math.nan, dtype=dtype, device=DEV)
    src[:, 5:5 + V] = x
    for start in (5, 3):                                           # rows of the same phase, and of another one
        out = torch.full((9, 1200), 7.0, dtype=dtype, device=DEV)
        d = api.sp_token_logprobs_grad(src[:, 5:5 + V], t, r.lse, gl, out=out[:, start:start + V])
        # (the row's sum is taken in the same order, wherever it starts)
        assert torch.equal(d, want)
        assert (out[:, :start] == 7).all() and (out[:, start + V:] == 7).all()
    x[3, 17] = math.nan
    x[1, 17] = math.inf
    r = api.sp_token_logprobs(x, t)
    d = api.sp_token_logprobs_grad(x, t, r.lse, gl)
    assert torch.isnan(d[[1, 3]]).all() and torch.equal(d[[0, 2, 4, 5, 6, 7, 8]], want[[0, 2, 4, 5, 6, 7, 8]])


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_padded_calibration_batch(dtype):
    """Rows before the first and behind the last sequence: no head outputs, and no part in the scores, the mask and the weights."""
    g = torch.Generator(device=DEV).manual_seed(4)
    n, d, heads, lead, tail = 300, 128, 4, 9, 55
    X = torch.randn(n, d, generator=g, device=DEV).to(dtype)
    W = (torch.randn(3 * d, d, generator=g, device=DEV) / math.sqrt(d)).to(dtype)
    Wo = torch.randn(d, d, generator=g, device=DEV) / math.sqrt(d)
    padded = torch.full((lead + n + tail, d), math.nan, dtype=dtype, device=DEV)
    padded[lead:lead + n] = X
    cu = lambda o: torch.tensor([o, o + 120, o + n], dtype=torch.int32, device=DEV)
    hold = [torch.full((lead + n + tail, d), math.nan, dtype=dtype, device=DEV) for _ in range(4)]      # what the allocator gives out next
    del hold
    H = pipeline.attention_head_outputs(padded, W, cu(lead), heads)
    alone = pipeline.attention_head_outputs(X, W, cu(0), heads)
    assert torch.equal(H[lead:lead + n], alone) and (H[:lead] == 0).all() and (H[lead + n:] == 0).all()
    a = pipeline.prune_attention_module(X, W, Wo, cu(0), heads, 2)
    b = pipeline.prune_attention_module(padded, W, Wo, cu(lead), heads, 2)
    assert torch.equal(a[0], b[0]) and torch.isfinite(b[1]).all() and torch.isfinite(b[2]).all()
    # sums of the same n products of storage type in another order: n 2^-23 of their magnitudes, which the squares of the scores equal
    assert ((a[2] - b[2]).abs() <= 2 * n * 2.0 ** -23 * a[2].abs()).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [1, 5, 77, 401, 777])
def test_one_row_that_ends_with_its_storage(dtype, K):
    """A single row has no pitch: what stands behind its K values belongs to somebody else."""
    g = torch.Generator(device=DEV).manual_seed(K)
    for T, N in ((1, 300), (1, 1), (7, 1)):
        x = torch.randn(T, (K + 7) // 8 * 8, generator=g, device=DEV).to(dtype)[:, :K] if T > 1 else torch.randn(1, K, generator=g, device=DEV).to(dtype)
        w = torch.randn(N, (K + 7) // 8 * 8, generator=g, device=DEV).to(dtype)[:, :K] if N > 1 else torch.randn(1, K, generator=g, device=DEV).to(dtype)
        y = api.sp_linear(x, w, out_dtype=torch.float32)
        want = x.double() @ w.double().T
        tol = (x.double().abs() @ w.double().abs().T) * K * 2.0 ** (-23 if dtype == torch.bfloat16 else -52) + 2.0 ** -23 * want.abs() + 1e-30
        assert ((y.double() - want).abs() <= tol).all()


def test_pipeline_functions_in_a_captured_graph():
    """With a status word of the caller nothing waits for the device; without one the wait is left out while a graph is captured."""
    g = torch.Generator(device=DEV).manual_seed(7)
    r = lambda *s: (torch.randn(*s, generator=g, device=DEV) / 8).bfloat16()
    X, Wqkv, W1, W2, Wg = r(200, 64), r(192, 64), r(96, 64), r(64, 96), r(96, 64)
    cu = torch.tensor([0, 150, 200], dtype=torch.int32, device=DEV)

    def layer(status):
        H = pipeline.attention_head_outputs(X, Wqkv, cu, 2, status=status)
        return pipeline.ffn_forward(H, W1, W2, Wg, residual=X, status=status)
    want = layer(None)
    for status in (api.new_status(), None):
        assert torch.equal(layer(status), want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer(status)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_a_wait_that_runs_out_under_a_pipeline_function_is_raised():
    """(With a budget of a few cycles ordinary waits run out, nothing is withheld.)"""
    g = torch.Generator(device=DEV).manual_seed(8)
    X = torch.randn(4096, 512, generator=g, device=DEV).bfloat16()
    Wqkv = (torch.randn(1536, 512, generator=g, device=DEV) / 22).bfloat16()
    cu = torch.tensor([0, 4096], dtype=torch.int32, device=DEV)
    want = pipeline.attention_head_outputs(X, Wqkv, cu, 8)
    status = api.new_status()
    assert api.lib().sp_set_wait_budget(8) == 0
    try:
        with pytest.raises(api.SpError) as e:
            pipeline.attention_head_outputs(X, Wqkv, cu, 8)
        assert e.value.code == 7
        pipeline.attention_head_outputs(X, Wqkv, cu, 8, status=status)
        assert int(status[0]) == 7
    finally:
        assert api.lib().sp_set_wait_budget(0) == 0
    assert torch.equal(pipeline.attention_head_outputs(X, Wqkv, cu, 8), want)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_gelu_keeps_its_relative_accuracy(out_dtype):
    """Down to where y Phi(y) leaves the normal range: within 2^-16 of its value (and half a step of storage)."""
    v = torch.cat([-torch.linspace(0.001, 13.0, 40000), torch.linspace(0.001, 13.0, 1001)]).to(DEV)
    for T in (1, 300):                                             # both forms
        x = torch.zeros(T, 16, dtype=torch.bfloat16, device=DEV)
        w = torch.zeros(v.numel(), 16, dtype=torch.bfloat16, device=DEV)
        y = api.sp_linear(x, w, bias=v, act=api.SP_LINEAR_GELU, out_dtype=out_dtype)
        want = v.double() * torch.special.log_ndtr(v.double()).exp()
        tol = (2.0 ** -16 + HALF[out_dtype] * (1 + 2.0 ** -16)) * want.abs() + 2.0 ** -126
        err = (y.double() - want).abs()
        assert (err <= tol).all(), (float((err / tol).max()), float(v[(err / tol).amax(0).argmax()]))


@pytest.mark.parametrize("q,k", [([1, 1], [700, 40]), ([300], [300])])     # single tokens; tiles of many rows
@pytest.mark.parametrize("dtype", DTYPES)
def test_scaled_logits_beyond_fp32_are_not_taken_for_a_mask(dtype, q, k):
    """scale <q, k> = +2^136 at every key: beyond fp32.  No probability can be told, so the rows are NaN: not 0, which says that a row sees
    no key."""
    Q, K, V = att.inputs(sum(q), sum(k), 2, 2, 64, dtype)
    Q.zero_()
    K.zero_()
    Q[:, ::64], K[:, ::64] = 2.0 ** 60, 2.0 ** 66
    o, lse = api.sp_attention(Q, K, V, att.cu(q), att.cu(k), 2, scale=2.0 ** 10, want_lse=True)
    assert torch.isnan(o).all() and not (lse == -math.inf).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dh", [64, 72])
@pytest.mark.parametrize("q", [[1] * 100 + [500] + [1] * 60, [0] * 90 + [600, 1] + [0] * 40, [3000] + [1] * 255])
def test_one_long_sequence_among_many_short_or_empty_ones(dtype, dh, q):
    """By the average these are few rows: the kernels that stream keys past some rows take the long sequence tile by tile."""
    k = [n if n > 1 else (37 * i) % 301 for i, n in enumerate(q)]
    Q, K, V = att.inputs(sum(q), sum(k), 2, 2, dh, dtype)
    assert sum(q) <= 16 * len(q)
    att.check(Q, K, V, q, k, 2, 2)
    att.check(Q, K, V, q, k, 2, 2, causal=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv", [(64, 1), (40, 2), (96, 1)])
def test_groups_wider_than_a_few_row_tile(dtype, heads, kv):
    """Slots of which most are empty: few rows on average, and more heads to a key head than a tile of them has rows."""
    q, k = [0] * 200, [0] * 200
    for at, n in ((3, 700), (77, 1), (140, 2100), (199, 64)):
        q[at], k[at] = 1, n
    q[150], k[150] = 2, 65
    Q, K, V = att.inputs(sum(q), sum(k), heads, kv, 64, dtype, seed=heads)
    assert sum(q) * heads // kv <= 16 * len(q)
    att.check(Q, K, V, q, k, heads, kv)
