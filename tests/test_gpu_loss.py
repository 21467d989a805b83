"""sp_token_logprobs and sp_token_logprobs_grad against the definitions in 64 bits.

Tolerances.  z = scale logit is formed from a scale rounded three times (3 half steps of 2^-24 of |z|, with the fused
multiply-add's own rounding 4); every exponential is off by its argument's rounding (2^-24 |z - max|, within 2 max|z|) and
the instruction's 2^-22; a thread adds n = V / 32 (rows of up to 4096) or V / 256 values and 9 joins follow, one step each:
lse within e = 2^-24 (12 max|z| + n + 64), logp within twice that.  The entropy is log s - w / s with w a sum of terms
t 2^t, t = log2 p - log2 p_max: the share of a relative error e of its terms is e E|t|, and E|t| <= 2 (entropy + 1); the
floor on t (-10000) is beyond what 2^t can represent."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def logits_of(T, V, dtype, seed=0, pitch=None, start=0, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = spread * torch.randn(T, V, generator=g, device=DEV)
    buf = torch.zeros(T, (pitch or V) + start, dtype=dtype, device=DEV)[:, start:start + V]
    buf.copy_(x)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    return buf, targets


def reference(x, targets, scale):
    z = x.double() * scale
    lse = torch.logsumexp(z, 1)
    empty = (z == -math.inf).all(1)
    lp = z - torch.where(empty, 0.0, lse)[:, None]
    p = torch.where(empty[:, None], 0.0, lp.exp())
    H = -torch.where(p > 0, p * lp, 0.0).sum(1)
    logp = None
    if targets is not None:
        logp = torch.where(targets < 0, 0.0, lp.gather(1, targets.clamp_min(0)[:, None]).squeeze(1))
        logp = torch.where(empty & (targets >= 0), -math.inf, logp)
    V = x.shape[1]
    zmax = torch.where(z.abs() < 1e30, z.abs(), 0.0).amax(1)       # (masked ones do not enter)
    e = 2.0 ** -24 * (12 * zmax + V / (32 if V <= 4096 else 256) + 64)
    return lse, logp, H, lp, p, e


def same_or_near(got, want, tol):
    got = got.double()
    inf = torch.isinf(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[inf], want[inf])
    fine = torch.isfinite(want)
    assert ((got - want).abs() <= tol)[fine].all(), float(((got - want).abs() / tol)[fine].max())


def check(x, targets, scale=1.0, n_alts=0, status=None):
    r = api.sp_token_logprobs(x, targets, n_alts=n_alts, scale=scale, status=status)
    lse, logp, H, lp, p, e = reference(x, targets, scale)
    same_or_near(r.lse, lse, e)
    if targets is not None:
        same_or_near(r.logp, logp, 2 * e)
    same_or_near(r.entropy, H, 4 * e * (1 + H))
    if n_alts:
        order = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :n_alts]
        assert torch.equal(r.alt_ids.long(), order)
        want = lp.gather(1, order)
        same_or_near(r.alt_logp, want, (2 * e)[:, None].expand_as(want))
    return r


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (1, 7), (9, 31), (17, 255), (8, 1000), (33, 4096), (5, 4097), (1, 32000),
                                 (2, 50257), (40, 50257), (700, 9001), (300, 8192), (1, 262147)])
def test_sizes(dtype, T, V):
    x, t = logits_of(T, V, dtype, seed=V)
    t[T // 2] = -100
    check(x, t, n_alts=min(5, V))
    check(x, t, scale=0.37)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_alts", [1, 2, 8, 20, 31, 32])
@pytest.mark.parametrize("V", [32, 3001, 30011])
def test_alternatives_with_ties(dtype, n_alts, V):
    """Values from a short list, so that most are equal: the lower index wins; zeros of both signs are equal."""
    g = torch.Generator(device=DEV).manual_seed(n_alts)
    vals = torch.tensor([0.0, -0.0, 1.5, 1.5, -3.0, 2.0, 2.0, -math.inf], device=DEV)
    x = vals[torch.randint(0, 8, (6, V), generator=g, device=DEV)].to(dtype)
    x[1] = 2.0                                                     # all equal
    x[2] = torch.arange(V, device=DEV).to(dtype)                   # rising: every value enters the list
    x[3] = -torch.arange(V, device=DEV).to(dtype)
    x[4] = -math.inf
    x[4, V // 2] = 0.25
    x[5] = -math.inf                                               # nothing at all
    check(x, torch.full((6,), V // 2, device=DEV), n_alts=n_alts)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [513, 40001])
def test_not_a_number_and_infinities(dtype, V):
    x, t = logits_of(5, V, dtype)
    t[:] = 7
    x[0, 100] = math.nan
    x[1, 100] = math.inf
    x[2, 100:] = -math.inf
    x[3, 7] = -math.inf                                            # the target itself
    r = api.sp_token_logprobs(x, t, n_alts=3)
    for v in (r.lse, r.logp, r.entropy):
        assert torch.isnan(v[:2]).all()
    assert r.logp[3] == -math.inf
    check(x[2:], t[2:], n_alts=3)
    want = torch.sort(torch.nan_to_num(x[0].double(), nan=-math.inf), descending=True, stable=True).indices[:3]
    assert torch.equal(r.alt_ids[0].long(), want) and r.alt_ids[1, 0] == 100
    y = torch.full((1, 5), math.nan, dtype=dtype, device=DEV)      # only the indices are left
    y[0, 3] = -math.inf
    assert api.sp_token_logprobs(y, None, n_alts=5).alt_ids.tolist() == [[3, 0, 1, 2, 4]]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 9001])
def test_masks_of_the_lowest_value(dtype, V):
    """A mask may be the type's lowest number instead of -infinity.  A row of nothing else is a uniform one: the lse is that number (log V
    is lost beside it), the log probabilities are -log V."""
    low = torch.finfo(dtype).min
    x, t = logits_of(4, V, dtype)
    x[0] = low
    x[1, 3:] = low
    x[2, ::2] = low
    t[:] = 1
    for scale in (1.0, 0.5):
        r = api.sp_token_logprobs(x, t, scale=scale, n_alts=3)
        assert abs(float(r.logp[0]) + math.log(V)) < 1e-5 and abs(float(r.entropy[0]) - math.log(V)) < 1e-4
        assert float(r.lse[0]) == pytest.approx(low * scale, rel=1e-6) and r.alt_ids[0].tolist() == [0, 1, 2]
        check(x[1:], t[1:], scale=scale, n_alts=3)
    hidden = x.clone()
    hidden[1, 3:] = -math.inf
    hidden[2, ::2] = -math.inf
    a, b = api.sp_token_logprobs(x[1:], t[1:]), api.sp_token_logprobs(hidden[1:], t[1:])
    assert torch.equal(a.lse, b.lse) and torch.equal(a.logp, b.logp)
    assert (a.entropy - b.entropy).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", DTYPES)
def test_targets_that_are_none(dtype):
    x, t = logits_of(6, 300, dtype)
    t[0], t[1], t[2], t[3] = -1, -100, 300, 1 << 40
    status = api.new_status()
    r = api.sp_token_logprobs(x, t, status=status)
    assert (r.logp[:2] == 0).all() and torch.isnan(r.logp[2:4]).all() and torch.isfinite(r.logp[4:]).all()
    code, row = status.tolist()[:2]
    assert code == 2 and row in (2, 3)
    assert api.sp_token_logprobs(x, None).logp is None
    d = api.sp_token_logprobs_grad(x, t, r.lse, torch.ones(6, device=DEV))
    assert (d[:4] == 0).all() and (d[4:] != 0).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pitch,start", [(1300, 0), (1003, 1), (1001, 5), (1009, 7)])
def test_pitches_and_starts(dtype, pitch, start):
    x, t = logits_of(20, 1001, dtype, pitch=pitch, start=start)
    check(x, t, n_alts=4)
    grad_check(x, t, 1.0, True)
    out = torch.full((20, 1200), 7.0, dtype=dtype, device=DEV)
    grad_check(x, t, 1.0, True, out=out[:, 3:1004])
    assert (out[:, :3] == 7).all() and (out[:, 1004:] == 7).all()


def grad_check(x, t, scale, with_entropy, out=None):
    T, V = x.shape
    g = torch.Generator(device=DEV).manual_seed(9)
    gl = torch.randn(T, generator=g, device=DEV)
    gh = torch.randn(T, generator=g, device=DEV) if with_entropy else None
    r = api.sp_token_logprobs(x, t, scale=scale)
    before = x.clone()
    d = api.sp_token_logprobs_grad(x, t, r.lse, gl, entropy=r.entropy if with_entropy else None, g_entropy=gh, scale=scale,
                                   out=out)
    u = before.double() * scale - r.lse.double()[:, None]
    p = u.exp()
    told = (t >= 0) & (t < V)
    one = torch.zeros(T, V, dtype=torch.float64, device=DEV)
    one[torch.arange(T, device=DEV)[told], t[told]] = 1.0
    a = torch.where(told, gl.double(), 0.0)[:, None]
    h = gh.double()[:, None] if with_entropy else torch.zeros(T, 1, dtype=torch.float64, device=DEV)
    H = r.entropy.double()[:, None]
    pu = torch.where(p > 0, p * u, 0.0)
    want = scale * (a * (one - p) - h * (pu + p * H))
    # p: the argument's roundings, 2^-23 |u| with log2(e), and the instruction's 2^-22; two multiplications more; one rounding.
    # The scale is held in 32 bits: u itself is off by 2^-24 |z| and, after the addition, 2^-24 |u|, and the derivative of
    # p (a + h (u + H)) with respect to u is p (a + h (u + H + 1)) -- where u is near 0 that is no small share of p u.
    mag = torch.where(p > 0, u.abs(), 0.0)
    rel = mag * 2.0 ** -22 + 2.0 ** -20
    e_u = 2.0 ** -24 * (torch.where(p > 0, (before.double() * scale).abs(), 0.0) + mag)
    tol = scale * rel * (p * a.abs() + h.abs() * (pu.abs() + p * H)) + HALF[x.dtype] * want.abs() + 2.0 ** -23 * scale * a.abs() * one
    tol = tol + scale * e_u * p * (a.abs() + h.abs() * (mag + H + 1))
    # (what a product below 2^-126 becomes)
    assert ((d.double() - want).abs() <= tol + 1e-37).all(), float(((d.double() - want).abs() / (tol + 1e-37)).max())
    return d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_entropy", [False, True])
@pytest.mark.parametrize("T,V", [(1, 1), (5, 6), (3, 33), (130, 1000), (7, 50257), (64, 8192)])
def test_gradient(dtype, with_entropy, T, V):
    x, t = logits_of(T, V, dtype, seed=T)
    if T > 2:
        t[1] = -1
    grad_check(x, t, 1.0, with_entropy)
    grad_check(x, t, 1.7, with_entropy)
    want = grad_check(x, t, 0.6, with_entropy)
    got = grad_check(x, t, 0.6, with_entropy, out=x)               # in place
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)


def test_gradient_of_the_entropy_alone_and_masked_logits():
    x, t = logits_of(8, 777, torch.float32)
    x[:, ::3] = -math.inf
    x[5] = -math.inf
    r = api.sp_token_logprobs(x, t)
    d = api.sp_token_logprobs_grad(x, t, r.lse, torch.ones(8, device=DEV), entropy=r.entropy, g_entropy=torch.ones(8, device=DEV))
    assert torch.isfinite(d).all() and (d[5] == 0).all()
    hidden = x == -math.inf
    hidden[torch.arange(8, device=DEV), t] = False
    assert (d[hidden] == 0).all()
    y = x.clone()
    y[5] = 1.0
    r = api.sp_token_logprobs(y)
    d = api.sp_token_logprobs_grad(y, None, r.lse, None, entropy=r.entropy, g_entropy=torch.ones(8, device=DEV))
    assert torch.isfinite(d).all() and d.double().sum(1).abs().max() < 1e-5


def test_gradient_against_differences():
    """Central differences of the forward call in fp32 storage: the quotient's error is h^2 / 6 times a third derivative (within
    scale^3 <= 1 here, weighted by |g| <= 1) plus two forward errors of at most 2^-20 over 2 h."""
    T, V, h = 4, 50, 2.0 ** -6
    x, t = logits_of(T, V, torch.float32, spread=1.0)
    gl, gh = torch.tensor([1.0, -0.5, 0.25, 0.0], device=DEV), torch.tensor([0.0, 0.5, -1.0, 1.0], device=DEV)
    r = api.sp_token_logprobs(x, t)
    d = api.sp_token_logprobs_grad(x, t, r.lse, gl, entropy=r.entropy, g_entropy=gh)
    f = lambda y: (lambda q: gl * q.logp + gh * q.entropy)(api.sp_token_logprobs(y, t)).double()
    for v in range(V):
        up, down = x.clone(), x.clone()
        up[:, v] += h
        down[:, v] -= h
        num = (f(up) - f(down)) / (2 * h)
        assert (num - d[:, v].double()).abs().max() < 6 * h * h + 2.0 ** -20 / h


@pytest.mark.parametrize("dtype", DTYPES)
def test_another_stream_capture_and_repeatability(dtype):
    x, t = logits_of(3, 70001, dtype)                              # a cluster per row
    want = check(x, t, n_alts=6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = api.sp_token_logprobs(x, t, n_alts=6)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    gl = torch.ones(3, device=DEV)
    with torch.cuda.graph(graph):
        c = api.sp_token_logprobs(x, t, n_alts=6)
        d = api.sp_token_logprobs_grad(x, t, c.lse, gl)
    graph.replay()
    torch.cuda.synchronize()
    for r2 in (r, c):
        for a, b in ((r2.logp, want.logp), (r2.lse, want.lse), (r2.entropy, want.entropy), (r2.alt_ids, want.alt_ids),
                     (r2.alt_logp, want.alt_logp)):
            assert torch.equal(a, b)
    assert torch.equal(d, api.sp_token_logprobs_grad(x, t, want.lse, gl))


def test_offsets_beyond_32_bits():
    T, V = 33000, 65536                                            # 2.16e9 logits
    x = torch.zeros(T, V, dtype=torch.bfloat16, device=DEV)
    x[-1, -5] = 20.0
    t = torch.full((T,), V - 5, device=DEV)
    r = api.sp_token_logprobs(x, t, n_alts=1)
    assert abs(float(r.logp[-1]) - (20.0 - math.log(math.exp(20.0) + V - 1))) < 1e-5 and int(r.alt_ids[-1]) == V - 5
    d = api.sp_token_logprobs_grad(x, t, r.lse, torch.ones(T, device=DEV), out=x)
    assert abs(float(d[-2, -5]) - (1 - 1 / V)) < 2.0 ** -8 and abs(float(d[-2, 0]) * V + 1) < 2.0 ** -7
