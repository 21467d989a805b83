"""The norm, the 8-bit projections and the paged cache as layers use them: prompts by chunks, then tokens one by one."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api, pipeline

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def freqs(n):
    return 10000.0 ** (-2.0 * torch.arange(n // 2, device=DEV).float() / n)


def turn(x, position, f, neighbours=False):
    """x [n, heads, dh] in 64 bits."""
    n = f.numel()
    angle = position.double()[:, None, None] * f.double()
    c, s, out = angle.cos(), angle.sin(), x.clone()
    at, bt = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if neighbours else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., at], x[..., bt]
    out[..., at], out[..., bt] = a * c - b * s, b * c + a * s
    return out


def attend(q, k, v, kv):
    """Causal attention in 64 bits, the last query sees every key: q [n, heads, dh], k, v [m, kv, dh]."""
    n, m, g, dh = q.shape[0], k.shape[0], q.shape[1] // kv, q.shape[2]
    z = torch.einsum("iagd,jad->agij", q.view(n, kv, g, dh), k) * dh ** -0.5
    z = z.masked_fill(torch.arange(m, device=DEV)[None, :] > torch.arange(n, device=DEV)[:, None] + m - n, -math.inf)
    return torch.einsum("agij,jad->iagd", torch.softmax(z, 3), v).reshape(n, kv * g, dh)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("turned", [64, 32])
def test_head_outputs_with_positions(neighbours, turned):
    """fp32: the projections' sums are in 64 bits, so that logits are off by little more than the roundings of q, k and the angles' cosines (2^-22 of
    |q| |k|, below 2^-18 here) and results by 2^-16 of the largest value."""
    heads, kv, dh, d = 4, 2, 64, 96
    lens = [37, 1, 100]
    N = sum(lens) + 3
    X = torch.randn(N, d, generator=gen(1), device=DEV)
    W = torch.randn((heads + 2 * kv) * dh, d, generator=gen(2), device=DEV) / d ** 0.5
    cu = torch.tensor([0, 37, 38, 138], dtype=torch.int32, device=DEV)
    H = pipeline.attention_head_outputs(X, W, cu, heads, kv, inv_freq=freqs(turned), neighbours=neighbours)
    assert (H[138:] == 0).all()
    qkv = (X.double() @ W.double().t()).view(N, -1, dh)
    at = 0
    for n in lens:
        rows, place = qkv[at:at + n], torch.arange(n, device=DEV)
        q, k = (turn(x, place, freqs(turned), neighbours) for x in (rows[:, :heads], rows[:, heads:heads + kv]))
        want = attend(q, k, rows[:, heads + kv:], kv).flatten(1)
        assert (H[at:at + n].double() - want).abs().max() <= 2.0 ** -16 * rows[:, heads + kv:].abs().max()
        at += n


@pytest.mark.parametrize("four", [False, True])
def test_chunks_and_tokens_through_a_cache(four):
    """fp32 activations, steps of all sizes: every step's head outputs are attention over what the cache holds (sp_cache_read), for texts that come,
    grow and go.  fp32 throughout: results within 2^-16 of the largest value."""
    heads, kv, dh = 8, 2, 64
    cache = pipeline.KvCache(1, 80, 16, kv, dh, four)
    f, g = freqs(dh), gen(3)
    steps = [(["a", "b"], [40, 7]), (["b", "a", "c"], [1, 1, 90]), (["a", "b", "c"], [1, 1, 1]), (["c"], [200]), (["b", "c"], [130, 0]),
             (["d", "a", "b", "c"], [17, 3, 1, 2])]
    for texts, new in steps:
        if "d" in texts:
            cache.close("a")                                     # (starts anew on pages that were others')
        step = cache.step(texts, new)
        N = sum(new)
        qkv = torch.randn(N + 2, (heads + 2 * kv) * dh, generator=g, device=DEV)
        before = qkv.clone()
        H = pipeline.cached_attention(qkv, cache.layers[0], step, heads, kv, f)
        assert (H[N:] == 0).all()
        lens = [cache.tokens(t) for t in texts]
        cu_all = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
        K, V = api.sp_cache_read(cache.layers[0], cu_all, step.table, step.lens, sum(lens), F32)
        at = 0
        for s, (n, m) in enumerate(zip(new, lens)):
            rows = before[at:at + n].double().view(n, heads + 2 * kv, dh)
            place = torch.arange(m - n, m, device=DEV)
            q = turn(rows[:, :heads], place, f)
            k, v = (x[int(cu_all[s]):int(cu_all[s + 1])].double().view(m, kv, dh) for x in (K, V))
            if n and step.fresh:
                k, v = turn(rows[:, heads:heads + kv], place, f), rows[:, heads + kv:]
            elif n:                                              # what went in is what came out, to the cache's steps
                held = (k[m - n:] - turn(rows[:, heads:heads + kv], place, f)).abs().max()
                assert held <= (0.4 if four else 2.0 ** -6)
            if n:
                want = attend(q, k, v, kv).flatten(1)
                assert (H[at:at + n].double() - want).abs().max() <= 2.0 ** -16 * v.abs().max()
            at += n


def layer(d, heads, kv, dh, k, seed, eight, gated=True, dtype=BF):
    g = gen(seed)
    def w(rows, cols):
        return torch.randn(rows, cols, generator=g, device=DEV) / cols ** 0.5
    up, down, gate, _ = pipeline.kept_ffn_weights((torch.rand(2 * k, generator=g, device=DEV).argsort() < k).to(torch.uint8), w(2 * k, d),
                                                  w(d, 2 * k) * 2 ** 0.5, w(2 * k, d) if gated else None, dtype=dtype)
    wqkv, wo = w((heads + 2 * kv) * dh, d).to(dtype), w(d, heads * dh).to(dtype)
    if eight:
        wqkv, up, gate = (None if x is None else pipeline.weights_8bit(x) for x in (wqkv, up, gate))
    norm = lambda: 1 + 0.1 * torch.randn(d, generator=g, device=DEV)
    return pipeline.LayerWeights(norm(), wqkv, wo, norm(), up, down, gate, heads, kv, freqs(dh))


def run(layers, cache, texts, chunks, inputs):
    """Streams of the texts, the chunks [(new tokens of each text), ...] one step each; [tokens of all texts in order]."""
    done, out = [0] * len(texts), [[] for _ in texts]
    for new in chunks:
        step = cache.step(texts, new)
        x, h = torch.cat([inputs[t][a:a + n] for t, a, n in zip(range(len(texts)), done, new)]), None
        for w, pages in zip(layers, cache.layers):
            x, h = pipeline.layer_forward(x, h, w, pages, step)
        r = api.sp_rms_norm(x, None, residual=h)
        at = 0
        for t, n in enumerate(new):
            out[t].append(r.Y[at:at + n])
            at += n
            done[t] += n
    return torch.cat([torch.cat(o) for o in out])


def plain(layers, x, dh):
    """One text through the layers in 64 bits."""
    full = lambda w: (w[0].double() * w[1].double()[:, None]) if isinstance(w, tuple) else w.double()
    norm = lambda h, w: h / (h.square().mean(1, keepdim=True) + 1e-5).sqrt() * w.double()
    h, place = x.double(), torch.arange(x.shape[0], device=DEV)
    for w in layers:
        qkv = (norm(h, w.norm_attn) @ full(w.wqkv).t()).view(x.shape[0], -1, dh)
        q, k = (turn(y, place, w.inv_freq) for y in (qkv[:, :w.n_heads], qkv[:, w.n_heads:w.n_heads + w.n_kv_heads]))
        h = h + attend(q, k, qkv[:, w.n_heads + w.n_kv_heads:], w.n_kv_heads).flatten(1) @ w.wo.double().t()
        n = norm(h, w.norm_ffn)
        a = n @ full(w.up).t()
        a = torch.relu(a) if w.gate is None else torch.nn.functional.silu(n @ full(w.gate).t()) * a
        h = h + a @ w.down.double().t()
    return norm(h, torch.ones(h.shape[1], device=DEV))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("eight, four", [(False, False), (True, False), (False, True), (True, True)])
def test_layers_token_by_token(eight, four, gated):
    """Two layers, FFN modules pruned to odd widths, two texts by chunks and tokens, against the formula in 64 bits on the same weights.  Of a layer's
    about ten roundings on the way of a value each leaves at most half a step, 2^-8, of a part of the stream, and 8-bit activations 2^-4 of one
    operand of each of two products, uniform and independent over the hundred and more terms of a sum, whose mean square is a third of that square:
    2 layers x 10 x 2^-8 / sqrt 3 in a row, and sqrt(2 layers x 2) 2^-4 / sqrt 3; a cache of 4 bits is off by half a step of about a third of a
    value's deviation, 0.1 of it in the mean square, in keys and in values of each layer."""
    d, heads, kv, dh, k = 256, 4, 2, 64, 333
    layers = [layer(d, heads, kv, dh, k, 10 + i, eight, gated) for i in range(2)]
    inputs = [torch.randn(n, d, generator=gen(20 + n), device=DEV).to(BF) for n in (60, 45)]
    want = torch.cat([plain(layers, x, dh) for x in inputs])
    cache = pipeline.KvCache(2, 20, 16, kv, dh, four)
    got = run(layers, cache, ["a", "b"], [(30, 40), (1, 1), (25, 0)] + [(1, 1)] * 4, inputs)
    off = 20 * 2.0 ** -8 / 3 ** 0.5 + (2 * 2.0 ** -4 / 3 ** 0.5 if eight else 0.0) + (0.1 * 2 * 2 ** 0.5 if four else 0.0)
    rel = ((got.double() - want).norm() / want.norm()).item()
    assert rel <= off, rel
    whole = run(layers, pipeline.KvCache(2, 20, 16, kv, dh, four), ["a", "b"], [(60, 45)], inputs)
    assert ((whole.double() - want).norm() / want.norm()).item() <= off


def test_layers_in_fp32():
    """fp32 activations and weights, keys and values in 16 bits: half a step of 2^-8 in keys and values of a layer, uniform (a third of the square), and the
    rest below."""
    d, heads, kv, dh, k = 192, 3, 3, 64, 101
    layers = [layer(d, heads, kv, dh, k, 30 + i, False, True, F32) for i in range(2)]
    x = [torch.randn(50, d, generator=gen(40), device=DEV)]
    got = run(layers, pipeline.KvCache(2, 8, 16, kv, dh), ["a"], [(20,), (29,), (1,)], x)
    want = plain(layers, x[0], dh)
    assert ((got.double() - want).norm() / want.norm()).item() <= 4 * 2.0 ** -8 / 3 ** 0.5
    whole = run(layers, pipeline.KvCache(2, 8, 16, kv, dh), ["a"], [(50,)], x)
    assert (whole.double() - want).abs().max() <= 2.0 ** -14 * want.abs().max()


def test_loss_of_a_normed_stream_and_its_gradients():
    """token_loss with the norm before the head, in fp32, against autograd in 64 bits: sums over 500 words and 48 channels in fp32 leave below 2^-14 of the
    largest gradient."""
    N, d, V = 70, 48, 500
    h = torch.randn(N, d, generator=gen(50), device=DEV) * 3
    W = torch.randn(V, d, generator=gen(51), device=DEV) / d ** 0.5
    w = 1 + 0.2 * torch.randn(d, generator=gen(52), device=DEV)
    t = torch.randint(0, V, (N,), generator=gen(53), device=DEV)
    t[::9] = -1
    r = pipeline.token_loss(h, W, t, token_chunk=32, with_grad=True, norm_weight=w)
    a, b, c = (x.double().requires_grad_() for x in (h, W, w))
    y = a / (a.square().mean(1, keepdim=True) + 1e-5).sqrt() * c
    loss = torch.nn.functional.cross_entropy(y @ b.t(), t, ignore_index=-1)
    loss.backward()
    assert abs(r.nll / r.tokens - loss.item()) < 1e-5
    for got, want in ((r.d_hidden, a.grad), (r.d_W, b.grad), (r.d_norm, c.grad)):
        assert (got.double() - want).abs().max() <= 2.0 ** -14 * want.abs().max()
    assert pipeline.token_loss(h, W, t, norm_weight=w).nll == pytest.approx(r.nll, rel=1e-6)
    assert r.d_norm.shape == (d,) and pipeline.token_loss(h, W, t, with_grad=True).d_norm is None


def test_a_decoding_step_captured_into_a_graph():
    """A layer's calls for one token of each text replay with the lengths and pages that the buffers hold then; status words are the caller's."""
    heads, kv, dh = 4, 2, 64
    cache = pipeline.KvCache(1, 40, 16, kv, dh, True)
    g = gen(60)
    first = cache.step(["a", "b"], [40, 9])
    pipeline.cached_attention(torch.randn(49, 512, generator=g, device=DEV).to(BF), cache.layers[0], first, heads, kv, freqs(dh))
    table = torch.full((2, 8), -1, dtype=torch.int32, device=DEV)
    lens, cu = torch.zeros(2, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    qkv, word = torch.zeros(2, 512, dtype=BF, device=DEV), api.new_status()
    held = pipeline.CacheStep(cu, lens, table, 0, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step = cache.step(["a", "b"], [1, 1])
        table[:, :step.table.shape[1]], lens[:] = step.table, step.lens
        x = torch.randn(2, 512, generator=g, device=DEV).to(BF)
        qkv.copy_(x)
        want = pipeline.cached_attention(qkv, cache.layers[0], held, heads, kv, freqs(dh), status=word)
        graph, f = torch.cuda.CUDAGraph(), freqs(dh)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            H = pipeline.cached_attention(qkv, cache.layers[0], held, heads, kv, f, status=word)
    torch.cuda.synchronize()
    qkv.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(H, want)
    for _ in range(20):                                          # (over the end of a page)
        step = cache.step(["a", "b"], [1, 1])
        table.fill_(-1)
        table[:, :step.table.shape[1]], lens[:] = step.table, step.lens
        x = torch.randn(2, 512, generator=g, device=DEV).to(BF)
        qkv.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = H.clone()
        qkv.copy_(x)
        assert torch.equal(got, pipeline.cached_attention(qkv, cache.layers[0], held, heads, kv, f, status=word))
    assert word.tolist() == [0, 0, 0, 0]


def test_calls_on_another_stream_than_the_tensors_own():
    heads, kv, dh = 8, 2, 128
    cache = pipeline.KvCache(1, 300, 16, kv, dh, True)
    q = torch.randn(2100, (heads + 2 * kv) * dh, generator=gen(70), device=DEV).to(BF)
    pipeline.cached_attention(q.clone(), cache.layers[0], cache.step(["a"], [2100]), heads, kv, freqs(dh))
    step = cache.step(["a"], [1])
    want = pipeline.cached_attention(q[:1].clone(), cache.layers[0], step, heads, kv, freqs(dh))
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    torch.cuda.synchronize()
    for s in streams:                                            # side by side, each with the workspace of its own call
        with torch.cuda.stream(s):
            got.append(api.sp_cache_attention(api.sp_cache_append(None, q[:1, 1024:1280], None, step.cu, None, step.lens, Q=q[:1, :1024],
                                                                  inv_freq=freqs(dh), d_head=dh), cache.layers[0], step.cu, step.table,
                                              step.lens, heads)[0])
    torch.cuda.synchronize()
    for x in got:
        assert torch.equal(x, want)


@pytest.mark.parametrize("four", [False, True])
def test_steps_without_tokens(four):
    cache = pipeline.KvCache(1, 4, 16, 2, 64, four)
    for texts, new in (([], []), (["a"], [0]), (["a", "b"], [0, 0])):
        H = pipeline.cached_attention(torch.zeros(0, 512, device=DEV), cache.layers[0], cache.step(texts, new), 4, 2, freqs(64))
        assert H.shape == (0, 256)
    qkv = torch.randn(5, 512, generator=gen(80), device=DEV)
    pipeline.cached_attention(qkv.clone(), cache.layers[0], cache.step(["a", "b"], [0, 5]), 4, 2, freqs(64))
    for texts, new in ((["b"], [0]), (["a", "b"], [0, 0]), ([], [])):
        H = pipeline.cached_attention(torch.zeros(2, 512, device=DEV), cache.layers[0], cache.step(texts, new), 4, 2, freqs(64))
        assert H.shape == (2, 256) and (H == 0).all()


def test_an_output_of_another_dtype_is_refused():
    X = torch.randn(4, 64, device=DEV).to(BF)
    for asked, given in ((torch.float8_e4m3fn, BF), (BF, torch.float8_e4m3fn)):
        with pytest.raises(ValueError, match="out_dtype"):
            api.sp_rms_norm(X, out_dtype=asked, out=torch.empty(4, 64, dtype=given, device=DEV))
    assert api.sp_rms_norm(X, out=torch.empty(4, 64, dtype=torch.float8_e4m3fn, device=DEV)).scale.shape == (4,)


def test_loss_of_a_normed_stream_in_bf16():
    """bf16: the normed rows, the logits' and the gradients' roundings, half a step of 2^-8 each at most and uniform: below 2^-7 of a gradient's norm
    in all, as the norm's own gradient comes from the rounded d_hidden."""
    N, d, V = 64, 128, 300
    h = torch.randn(N, d, generator=gen(90), device=DEV).to(BF)
    W = (torch.randn(V, d, generator=gen(91), device=DEV) / d ** 0.5).to(BF)
    w = 1 + 0.2 * torch.randn(d, generator=gen(92), device=DEV)
    t = torch.randint(0, V, (N,), generator=gen(93), device=DEV)
    r = pipeline.token_loss(h, W, t, with_grad=True, norm_weight=w)
    a, b, c = (x.double().requires_grad_() for x in (h, W, w))
    y = a / (a.square().mean(1, keepdim=True) + 1e-5).sqrt() * c
    torch.nn.functional.cross_entropy(y @ b.t(), t).backward()
    for got, want in ((r.d_hidden, a.grad), (r.d_W, b.grad), (r.d_norm, c.grad)):
        assert ((got.double() - want).norm() / want.norm()).item() <= 2.0 ** -7
