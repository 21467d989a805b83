"""The operators together, as the pipeline uses them: calibration inputs through an attention module and a pruned FFN module, heads pruned
from the module's input, and the predictions scored with the gradient of the score.  Every stage is compared with the definition in 64 bits
on the stage's own inputs: storage rounds once per stage (bf16 half a step 2^-8, of the probabilities too; fp32 2^-24), sums of K terms are
off by at most K 2^-23 of the sum of magnitudes."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api, pipeline

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
LENGTHS = [130, 1, 77, 200]
N, D, HEADS, N_FFN, V = sum(LENGTHS), 256, 4, 640, 1003


def weights(dtype, heads=HEADS, kv=HEADS, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    dh = D // heads
    return dict(X=r(N, D).to(dtype), Wqkv=(r((heads + 2 * kv) * dh, D) / math.sqrt(D)).to(dtype), bqkv=0.1 * r((heads + 2 * kv) * dh),
                Wo=r(D, D) / math.sqrt(D), W1=r(N_FFN, D) / math.sqrt(D), W2=r(D, N_FFN) / math.sqrt(N_FFN),
                Wg=r(N_FFN, D) / math.sqrt(D), b1=0.1 * r(N_FFN), b2=0.1 * r(D), W_lm=(r(V, D) / math.sqrt(D)).to(dtype),
                cu=torch.tensor([sum(LENGTHS[:i]) for i in range(len(LENGTHS) + 1)], dtype=torch.int32, device=DEV))


def near(got, want, tol):
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (err <= tol).all(), float((err / tol).max())


def linear64(x, w, b=None):
    """x w^T + b and the sum of magnitudes times K 2^-23."""
    y, m = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    return (y + b.double() if b is not None else y), (m + 1) * (x.shape[1] + 2) * 2.0 ** -23


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv", [4, 1])
def test_head_outputs(dtype, kv):
    w = weights(dtype, kv=kv)
    dh = D // HEADS
    H = pipeline.attention_head_outputs(w["X"], w["Wqkv"], w["cu"], HEADS, kv, bias=w["bqkv"])
    qkv = api.sp_linear(w["X"], w["Wqkv"], bias=w["bqkv"])
    want, e = linear64(w["X"], w["Wqkv"], w["bqkv"])
    near(qkv, want, e + HALF[dtype] * want.abs())
    at = w["cu"].tolist()
    for s, n in enumerate(LENGTHS):
        rows = slice(at[s], at[s] + n)
        for h in range(HEADS):
            j = h // (HEADS // kv)
            part = lambda k: qkv[rows, k * dh:(k + 1) * dh].double()
            q, k, v = part(h), part(HEADS + j), part(HEADS + kv + j)
            z = (q @ k.T) / math.sqrt(dh)
            hidden = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
            e = ((q.abs() @ k.abs().T) / math.sqrt(dh) * (dh + 4) * 2.0 ** -23).masked_fill(hidden, 0).amax(1, keepdim=True)
            p = z.masked_fill(hidden, -math.inf).softmax(1)
            want = p @ v
            near(H[rows, h * dh:(h + 1) * dh], want, (HALF[dtype] + 2 * e + (n + 32) * 2.0 ** -23) * (p @ v.abs()) + HALF[dtype] * want.abs() + 1e-30)


def test_heads_pruned_from_the_module_input():
    """What prune_attention_heads finds on the same head outputs; the heads kept are those with the largest scores."""
    w = weights(torch.bfloat16)
    mask, W_new, scores, H, Ypre = pipeline.prune_attention_module(w["X"], w["Wqkv"], w["Wo"], w["cu"], HEADS, 2, token_chunk=256)
    m2, W2, s2 = pipeline.prune_attention_heads(H, Ypre, w["Wo"], HEADS, 2, token_chunk=256)
    assert torch.equal(mask, m2) and torch.equal(scores, s2) and int(mask.sum()) == 2
    assert torch.allclose(W_new, W2, rtol=1e-3, atol=1e-4)
    assert set(torch.topk(scores, 2).indices.tolist()) == set(torch.nonzero(mask).flatten().tolist())
    dh = D // HEADS
    pruned = (mask == 0).repeat_interleave(dh)
    assert (W_new[:, pruned] == 0).all() and torch.isfinite(W_new).all()
    want, e = linear64(H, w["Wo"].bfloat16())
    near(Ypre, want, e + HALF[torch.bfloat16] * want.abs())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kept", [1, 201, 640])
def test_pruned_ffn(dtype, gated, kept):
    w = weights(dtype)
    g = torch.Generator(device=DEV).manual_seed(kept)
    mask = torch.zeros(N_FFN, dtype=torch.uint8, device=DEV)
    mask[torch.randperm(N_FFN, generator=g, device=DEV)[:kept]] = 1
    up, down, gate, b1 = pipeline.kept_ffn_weights(mask, w["W1"], w["W2"], w["Wg"] if gated else None, w["b1"], dtype)
    assert up.shape == (kept, D) and down.shape == (D, kept) and down.stride(0) % (16 // dtype.itemsize) == 0
    y = pipeline.ffn_forward(w["X"], up, down, gate, b1, w["b2"], residual=w["X"])
    z, e = linear64(w["X"], up, b1)
    if gated:
        u, eu = linear64(w["X"], gate)
        z = z + 0.0
        first = z                                                  # rounded to storage before the gate multiplies it
        a = torch.nn.functional.silu(u) * first
        ea = torch.nn.functional.silu(u).abs() * (e + HALF[dtype] * first.abs()) + (1.1 * eu + 2.0 ** -16 * u.abs()) * (first.abs() + e) + HALF[dtype] * a.abs()
    else:
        a, ea = z.clamp_min(0), e + HALF[dtype] * z.abs()
    want = a @ down.double().T + w["b2"].double() + w["X"].double()
    tol = 1.02 * ea @ down.double().abs().T + (a.abs() @ down.double().abs().T + 1) * (kept + 2) * 2.0 ** -23
    near(y, want, tol + (HALF[dtype] + 2.0 ** -22) * want.abs() + 1e-30)


def loss64(hidden, W, targets):
    z = hidden.double() @ W.double().T
    lp = z.log_softmax(1)
    told = targets >= 0
    return lp, torch.where(told, lp.gather(1, targets.clamp_min(0)[:, None]).squeeze(1), 0.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("chunk", [64, 1000])
def test_token_loss_and_its_gradient(dtype, chunk):
    w = weights(dtype)
    g = torch.Generator(device=DEV).manual_seed(5)
    t = torch.randint(0, V, (N,), generator=g, device=DEV)
    t[::7] = -100
    r = pipeline.token_loss(w["X"], w["W_lm"], t, token_chunk=chunk, with_grad=True)
    # the logits are rounded to storage: half a step of the largest, on both terms of z_t - lse, and the sums of D products
    lp, want = loss64(w["X"], w["W_lm"], t)
    z, e = linear64(w["X"], w["W_lm"])
    ez = (e + HALF[dtype] * z.abs()).amax(1)
    near(r.logp, want, 2 * ez + 2.0 ** -24 * (12 * z.abs().amax(1) + V / 32 + 64) * 2)
    told = t >= 0
    assert r.tokens == int(told.sum()) and abs(r.nll + float(r.logp.double().sum())) < 1e-6 * abs(r.nll)
    assert abs(math.log(r.perplexity) - r.nll / r.tokens) < 1e-9
    # gradient: p moves by a factor within exp(+-2 ez); it is rounded to storage, then summed over the vocabulary (over the tokens)
    p = lp.exp()
    one = torch.zeros_like(p)
    one[torch.arange(N, device=DEV)[told], t[told]] = 1.0
    dz = torch.where(told[:, None], p - one, 0.0) / r.tokens
    edz = (torch.where(told[:, None], p, 0.0) * (2.1 * ez[:, None] + 2.0 ** -18) / r.tokens) + HALF[dtype] * dz.abs() * 1.1 + 1e-30
    Wd, X = w["W_lm"].double(), w["X"].double()
    dh = dz @ Wd
    near(r.d_hidden, dh, 1.02 * edz @ Wd.abs() + (dz.abs() @ Wd.abs()) * V * 2.0 ** -23 + HALF[dtype] * dh.abs() * 1.02 + 1e-30)
    dW = dz.T @ X
    near(r.d_W, dW, 1.02 * edz.T @ X.abs() + (dz.abs().T @ X.abs()) * (N + 8) * 2.0 ** -23 + 1e-30)
    again = pipeline.token_loss(w["X"], w["W_lm"], t, token_chunk=chunk)
    assert again.d_W is None and torch.equal(again.logp, r.logp)


def test_gradient_of_the_loss_against_differences():
    """fp32 storage: central differences of the mean loss in a few directions; the quotient is off by h^2 / 6 times a third derivative
    (within (2 |direction . W| max)^3 < 1 for these) plus the rounding of two sums, 2^-18 / h."""
    w = weights(torch.float32)
    t = torch.arange(N, device=DEV) % V
    r = pipeline.token_loss(w["X"], w["W_lm"], t, with_grad=True)
    g = torch.Generator(device=DEV).manual_seed(2)
    h = 2.0 ** -6
    for _ in range(4):
        d = torch.randn(N, D, generator=g, device=DEV) * 0.1
        up, down = (pipeline.token_loss(w["X"] + s * h * d, w["W_lm"], t) for s in (1, -1))
        num = (up.nll - down.nll) / (2 * h) / N
        assert abs(num - float((r.d_hidden.double() * d.double()).sum())) < h * h / 6 + 2.0 ** -18 / h


def test_targets_outside_the_vocabulary_are_refused():
    w = weights(torch.bfloat16)
    t = torch.zeros(N, dtype=torch.int64, device=DEV)
    t[3] = V
    with pytest.raises(api.SpError):
        pipeline.token_loss(w["X"], w["W_lm"], t)


def test_a_layer_after_its_pruning():
    """Algorithm 1's FFN part on the output of an attention module, then the pruned layer's output: finite, and nearer to the unpruned
    layer's than that of the same channels without recovery (the recovery minimises that distance on these tokens)."""
    w = weights(torch.bfloat16, seed=3)
    H = pipeline.attention_head_outputs(w["X"], w["Wqkv"], w["cu"], HEADS, bias=w["bqkv"])
    X1 = api.sp_linear(H, w["Wo"].bfloat16(), other=w["X"])
    res, _, _, _ = pipeline.prune_ffn_layers(lambda l: (X1, w["W1"], w["W2"]), 1, N_FFN, 0.4, 3, api.AdmmParams(rho=1e-3))
    res = res[0]
    full = pipeline.ffn_forward(X1, w["W1"].bfloat16(), w["W2"].bfloat16())
    up, down, _, _ = pipeline.kept_ffn_weights(res.mask, res.W1, res.W2)
    pruned = pipeline.ffn_forward(X1, up, down)
    up0, down0, _, _ = pipeline.kept_ffn_weights(res.mask, w["W1"], w["W2"])
    plain = pipeline.ffn_forward(X1, up0, down0)
    dist = lambda a: float((a.double() - full.double()).norm())
    assert torch.isfinite(pruned).all() and dist(pruned) < dist(plain)
