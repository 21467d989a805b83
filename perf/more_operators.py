"""The operators between the projections of a layer that is served from a paged cache, as cases of one call each.

  norm       residual added, root-mean-square norm, the result in the activations' type or in 8 bits with a scale per row
  norm_grad  its gradient, with the one that arrives at the sum through the residual stream
  linear8    a projection whose operands are held in 8 bits with a scale per row and per output, and what follows it in a layer
  append     queries and keys turned by their positions, keys and values put into the pages of a cache (16 bits, or 4 with a scale
             and an offset for every 64 channels), and read back as the values that they stand for
  paged      attention over such a cache: single new tokens, a few drafted ones, the next chunk of a prompt

Head layouts and widths are those of the repository's workloads (12 x 64, 32 x 64, 32 x 128 heads; widths 768 to 4096, FFN widths
cut by its sparsities, so that kept counts are odd), grouped key and value heads, page lengths and cache lengths are generic.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
E4M3_MAX = 448.0
GROUP = 64                    # channels that share a scale and an offset in a cache of 4 bits


def _norm(name, kind, T, d, **kw):
    c = dict(name=name, kind=kind, T=T, d=d, dtype="bf16", stream="bf16", residual=True, eight=False)
    c.update(kw)
    return c


def _lin(name, T, n_in, n_out, **kw):
    c = dict(name=name, kind="linear8", T=T, n_in=n_in, n_out=n_out, bias=False, act="none", other="none")
    c.update(kw)
    return c


def _append(name, new, before, heads, kv, dh, **kw):
    new, before = (" ".join(map(str, x)) for x in (new, before))      # tokens of the call, tokens there before, by sequence
    c = dict(name=name, kind="append", new=new, before=before, heads=heads, kv=kv, dh=dh, dtype="bf16", cache="4bit", page=64,
             turned=dh, pairs="halves")
    c.update(kw)
    return c


def _paged(name, q, k, heads, kv, dh, **kw):
    q, k = (" ".join(map(str, x)) for x in (q, k))                    # queries and keys, by sequence
    c = dict(name=name, kind="paged", q=q, k=k, heads=heads, kv=kv, dh=dh, dtype="bf16", cache="4bit", page=64, causal=True, tail=0,
             lse=True)
    c.update(kw)
    return c


def listed():
    return [
        # a few new tokens in the smallest model: latency alone
        _norm("norm_768_few", "norm", 4, 768),
        # the tokens of a chunk of prompts before an 8-bit projection: bound by reading x and the stream, writing the stream and 8 bits
        _norm("norm_8bit_16384x4096", "norm", 16384, 4096, eight=True),
        # gradient for a short batch in fp32, the smallest model
        _norm("norm_grad_500x768", "norm_grad", 500, 768, dtype="f32", stream="f32"),
        # gradient for four segments of 2048 tokens: bound by reading the stream and two gradients, writing one
        _norm("norm_grad_8192x4096", "norm_grad", 8192, 4096),
        # query, key and value projections of 16 single tokens, 32 heads of 128 on 8: bound by reading the weight once
        _lin("linear8_tokens_6144", 16, 4096, 6144),
        # gate branch of a gated module pruned to 30 %, a chunk of prompts: silu of the product times the up branch
        _lin("linear8_gate_3303", 16384, 4096, 3303, act="silu", other="mul"),
        # one new token of each of 64 texts, caches of many lengths: latency
        _append("append_tokens_4bit", [1] * 64, [37 + 517 * i for i in range(64)], 32, 8, 128),
        # prompts of very different lengths, one of them the end of a longer one, an empty one among them
        _append("append_prompts_4bit", [4096, 1, 2047, 333, 0, 3000, 977, 130], [0, 5, 0, 0, 0, 8192, 0, 1000], 32, 8, 128, page=16),
        # one new token against a short cache of 16 bits, the smallest model's heads: latency alone
        _paged("paged_token_768", [1], [777], 12, 12, 64, cache="16bit", page=16),
        # a batch of single tokens, caches of many lengths in 4 bits: bound by reading the caches
        _paged("paged_tokens_4bit", [1] * 16, [2048 + 1931 * i for i in range(16)], 32, 8, 128),
        # five drafted tokens of each of 12 texts to be verified, ragged cache of 16 bits, a padded end
        _paged("paged_drafts_16bit", [5, 5, 3, 5, 1, 5, 5, 2, 5, 4, 5, 5], [700 + 977 * i for i in range(12)], 32, 8, 64, cache="16bit",
               page=16, tail=7),
        # the next chunk of a long prompt against a cache of 4 bits: bound by the matrix products
        _paged("paged_chunk_4bit", [512], [16384], 32, 8, 128),
    ]


def _lengths(text):
    return [int(x) for x in text.split()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "linear8", "append", "paged", "paged"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "norm_grad"):
        d = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
        T = _log_int(rng, 1, min(32768, (16384 * 4096 if kind == "norm" else 8192 * 4096) // (2 * d)))
        return _norm(None, kind, T, d, dtype=dtype, stream=rng.choice([dtype, "f32"]), residual=rng.random() < 0.7,
                     eight=kind == "norm" and rng.random() < 0.5)
    if kind == "linear8":
        n_in, n_out = (_log_int(rng, 64, 6000) for _ in range(2))
        T = _log_int(rng, 1, min(16384, max(1, 16384 * 4096 * 3303 // (n_in * n_out))))
        return _lin(None, T, n_in, n_out, bias=rng.random() < 0.6, act=rng.choice(["none", "relu", "silu", "gelu"]),
                    other=rng.choice(["none", "add", "mul"]))
    cache = rng.choice(["4bit", "4bit", "16bit"])
    dh = rng.choice([64, 128] if cache == "4bit" else [64, 128, 80, 96])
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        n = _log_int(rng, 1, 64)
        new = [1] * n if rng.random() < 0.5 else [_log_int(rng, 1, 4096) - 1 for _ in range(n)]
        while len(new) > 1 and sum(new) * (heads + 2 * kv) * dh > 10000 * 48 * 128:
            new = new[:-1]
        new[0] = max(new[0], 1)
        before = [_log_int(rng, 1, 200000) - 1 for _ in new]
        return _append(None, new, before, heads, kv, dh, dtype=dtype, cache=cache, page=page,
                       turned=rng.choice([dh, dh, dh // 32 * 16, 0]), pairs=rng.choice(["halves", "neighbours"]))
    form = rng.choice(["tokens", "tokens", "drafts", "chunk"])
    if form == "chunk":
        n = _log_int(rng, 1, 4)
        q = [_log_int(rng, 1, 700) for _ in range(n)]
    else:
        n = _log_int(rng, 1, 64)
        q = [1 if form == "tokens" else rng.randint(1, 8) for _ in range(n)]
    k = [x + _log_int(rng, 1, 32768 if form == "tokens" else 8192) - 1 for x in q]
    while len(q) > 1 and (sum(k) * kv * dh > 16 * 16530 * 8 * 128 or sum(a * b for a, b in zip(q, k)) * heads * dh > 512 * 16384 * 32 * 128
                          or len(q) * max(q) * max(k) * heads > 1 << 29 or len(q) * max(k) * kv * dh > 1 << 30):
        q, k = q[:-1], k[:-1]
    return _paged(None, q, k, heads, kv, dh, dtype=dtype, cache=cache, page=page, causal=rng.random() < 0.8,
                  tail=rng.choice([0, 0, 1, 17]), lse=rng.random() < 0.7)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _wide(rows, cols, dtype):
    """[rows, cols] whose rows start on 16 bytes, as a program lays out activations of an odd width."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.zeros(rows, (cols + per - 1) // per * per, dtype=dtype, device=DEV)[:, :cols]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _table(g, pages_of, first_of):
    """Page table and number of pages: sequence s has pages first_of[s] .. pages_of[s] - 1 of its own, scattered over the pool as a
    program that allots and frees them leaves them; entries before those are of pages that the call does not touch."""
    n_pages = sum(p - f for p, f in zip(pages_of, first_of))
    order = torch.randperm(max(n_pages, 1), generator=g, device=DEV).int()
    table = torch.zeros(len(pages_of), max(max(pages_of), 1), dtype=torch.int32, device=DEV)
    at = 0
    for s, (p, f) in enumerate(zip(pages_of, first_of)):
        table[s, f:p] = order[at:at + p - f]
        at += p - f
    return table, max(n_pages, 1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    st = {"case": case}
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        T, d, dt, ds = case["T"], case["d"], DTYPES[case["dtype"]], DTYPES[case["stream"]]
        strong = 1.0 + 29.0 * (torch.rand(d, generator=g, device=DEV) < 0.005)      # outlier channels of the residual stream
        st["weight"] = 1.0 + 0.2 * normal(d)
        if kind == "norm":
            x = _wide(T, d, dt)
            x.copy_(normal(T, d))
            st["X"], st["R"] = x, None
            if case["residual"]:
                st["R"] = _wide(T, d, ds)
                st["R"].copy_(normal(T, d) * strong)
            return st
        st["H"], st["dY"], st["dH"] = _wide(T, d, ds), _wide(T, d, dt), None
        st["H"].copy_(normal(T, d) * strong)
        st["dY"].copy_(normal(T, d))
        st["rstd"] = st["H"].double().square().mean(1).add(EPS).rsqrt().float()
        if case["residual"]:
            st["dH"] = _wide(T, d, ds)
            st["dH"].copy_(normal(T, d))
        return st
    if kind == "linear8":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        for name, rows, spread in (("X", T, 1.0), ("W", n_out, n_in ** -0.5)):
            full = normal(rows, n_in) * spread
            if name == "X":
                full = full * (1.0 + 9.0 * (torch.rand(n_in, generator=g, device=DEV) < 0.005))
            scale = full.abs().amax(1).clamp_min(1e-30) / E4M3_MAX
            eight = _wide(rows, n_in, torch.float8_e4m3fn)
            eight.copy_((full / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX))
            st[name], st[name + "_scale"] = eight, scale
        st["bias"] = 0.1 * normal(n_out) if case["bias"] else None
        st["other"] = None
        if case["other"] != "none":
            st["other"] = _wide(T, n_out, torch.bfloat16)
            st["other"].copy_(normal(T, n_out))
        return st
    dt, heads, kv, dh, page = DTYPES[case["dtype"]], case["heads"], case["kv"], case["dh"], case["page"]
    four = case["cache"] == "4bit"
    strong = 1.0 + 3.0 * (torch.rand(dh, generator=g, device=DEV) < 0.03)      # a few strong channels in queries and keys
    if kind == "append":
        new, before = _lengths(case["new"]), _lengths(case["before"])
        after = [a + b for a, b in zip(new, before)]
        T = sum(new)
        q, k, v = heads * dh, kv * dh, kv * dh
        qkv = normal(max(T, 1), heads + 2 * kv, dh)                       # one matrix, as one projection leaves them
        qkv[:, :heads + kv] *= strong
        st["qkv"] = qkv.reshape(max(T, 1), q + k + v).to(dt)
        st["cu"], st["lens"] = _ints(_offsets(new)), _ints(after)
        st["table"], n_pages = _table(g, [-(-a // page) for a in after], [b // page for b in before])
        st["inv_freq"] = 10000.0 ** (-2.0 * torch.arange(case["turned"] // 2, device=DEV, dtype=torch.float32) / max(case["turned"], 1))
    else:
        q_len, k_len = _lengths(case["q"]), _lengths(case["k"])
        st["Q"] = (normal(sum(q_len) + case["tail"], heads, dh) * strong).reshape(-1, heads * dh).to(dt)
        st["cu_q"], st["lens"] = _ints(_offsets(q_len)), _ints(k_len)
        st["keys"] = sum(k_len)
        st["table"], n_pages = _table(g, [-(-a // page) for a in k_len], [0] * len(k_len))
        st["out"] = torch.zeros_like(st["Q"])                             # the caller's buffers: rows behind the last
        st["lse"] = torch.zeros(st["Q"].shape[0], heads, device=DEV) if case["lse"] else None      # sequence stay as they are
    for name in "kv":
        if four:
            st[name + "_pages"] = torch.zeros(n_pages, kv, page, dh // 2, dtype=torch.uint8, device=DEV)
            st[name + "_scale"] = torch.zeros(n_pages, kv, page, dh // GROUP, 2, dtype=torch.bfloat16, device=DEV)
        else:
            st[name + "_pages"], st[name + "_scale"] = torch.zeros(n_pages, kv, page, dh, dtype=torch.bfloat16, device=DEV), None
        if kind == "append":
            continue
        some = max(1, (1 << 24) // (kv * page * dh))
        for a in range(0, n_pages, some):                                 # values near the normal distribution, by groups of 64
            n = min(some, n_pages - a)
            if not four:
                st[name + "_pages"][a:a + n] = normal(n, kv, page, dh) * (strong if name == "k" else 1.0)
                continue
            ints = (normal(n, kv, page, dh) * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            st[name + "_pages"][a:a + n] = ints[..., 0::2] | (ints[..., 1::2] << 4)
            scale = 0.37 * (0.8 + 0.4 * torch.rand(n, kv, page, dh // GROUP, generator=g, device=DEV))
            st[name + "_scale"][a:a + n, ..., 0] = scale
            st[name + "_scale"][a:a + n, ..., 1] = -7.5 * scale + 0.1 * normal(n, kv, page, dh // GROUP)
    return st


# ------------------------------------------------------------------------------------------------- plain forms, 32 bits
def _plain_norm(st):
    c = st["case"]
    h = st["X"].float()
    if st["R"] is not None:
        h = h + st["R"].float()
    rstd = (h * h).mean(1, keepdim=True).add(EPS).rsqrt()
    y = h * rstd * st["weight"]
    out = {"rstd": rstd.squeeze(1)}
    if st["R"] is not None:
        out["H"] = h.to(st["R"].dtype)
    if c["eight"]:
        scale = y.abs().amax(1).clamp_min(1e-30) / E4M3_MAX
        out["Y"] = (y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        out["scale"] = scale
    else:
        out["Y"] = y.to(st["X"].dtype)
    return out


def _plain_norm_grad(st):
    dy, rstd = st["dY"].float(), st["rstd"][:, None]
    xhat = st["H"].float() * rstd
    wdy = dy * st["weight"]
    dx = rstd * (wdy - xhat * (wdy * xhat).mean(1, keepdim=True))
    if st["dH"] is not None:
        dx = dx + st["dH"].float()
    return {"dX": dx.to(st["H"].dtype), "dweight": (dy * xhat).sum(0)}


def _activate(y, act):
    if act == "relu":
        return y.clamp_min(0)
    if act == "silu":
        return y / (1 + (-y).exp())
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain_linear8(st):
    c = st["case"]
    y = torch.matmul(st["X"].float(), st["W"].float().t()) * st["X_scale"][:, None] * st["W_scale"]
    if st["bias"] is not None:
        y = y + st["bias"]
    y = _activate(y, c["act"])
    if c["other"] == "add":
        y = y + st["other"].float()
    elif c["other"] == "mul":
        y = y * st["other"].float()
    return {"Y": y.to(torch.bfloat16)}


def _turn(x, angle, pairs):
    """x [T, heads, dh] with its first 2 * angle.shape[1] channels turned by pairs."""
    n = angle.shape[1]
    if n == 0:
        return x
    cos, sin = angle.cos().to(x.dtype)[:, None], angle.sin().to(x.dtype)[:, None]
    a, b = (x[..., :n], x[..., n:2 * n]) if pairs == "halves" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((u, v), 2) if pairs == "halves" else torch.stack((u, v), 3).flatten(2)
    return torch.cat((turned, x[..., 2 * n:]), 2)


def _four_bits(x):
    """The values that 4 bits with a scale and an offset per group hold for x (in 64 bits: values stand next to the border of two)."""
    groups = x.view(x.shape[0], -1, GROUP)
    low, high = groups.amin(2, keepdim=True), groups.amax(2, keepdim=True)
    zero = low.bfloat16().double()
    scale = ((high - zero) / 15).bfloat16().double()
    n = torch.where(scale > 0, (groups - zero) / scale, torch.zeros_like(groups)).round().clamp(0, 15)
    return (n * scale + zero).view_as(x)


def _plain_append(st):
    c = st["case"]
    heads, kv, dh = c["heads"], c["kv"], c["dh"]
    cu, T = st["cu"].long(), st["qkv"].shape[0]
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True).clamp(max=cu.numel() - 2)
    position = row - cu[seq + 1] + st["lens"].long()[seq]
    angle = position.double()[:, None] * st["inv_freq"].double()          # (far positions: 32 bits would not hold the angle)
    x = st["qkv"].view(T, heads + 2 * kv, dh)
    q = _turn(x[:, :heads].float(), angle, c["pairs"]).reshape(T, heads * dh).to(x.dtype)
    k, v = x[:, heads:heads + kv], x[:, heads + kv:]
    if c["cache"] == "4bit":
        k = _four_bits(_turn(k.double(), angle, c["pairs"]).reshape(T, kv * dh))
        v = _four_bits(v.double().reshape(T, kv * dh))
    else:
        k = _turn(k.float(), angle, c["pairs"]).reshape(T, kv * dh).bfloat16()
        v = v.reshape(T, kv * dh).bfloat16()
    return {"Q": q, "K": k.to(x.dtype), "V": v.to(x.dtype)}


def _plain_paged(st):
    c = st["case"]
    heads, kv, dh, page = c["heads"], c["kv"], c["dh"], c["page"]
    q_len, k_len = _lengths(c["q"]), _lengths(c["k"])
    n, g, mq, mk = len(q_len), heads // kv, max(q_len), max(k_len)
    cu, lk = st["cu_q"].long(), st["lens"].long()
    lq = cu[1:] - cu[:-1]
    i = torch.arange(mq, device=DEV)
    at = (cu[:-1, None] + i).clamp(max=st["Q"].shape[0] - 1)               # rows beyond a sequence repeat some row, masked below
    q = st["Q"].float().view(-1, kv, g, dh)[at].permute(0, 2, 3, 1, 4).reshape(n, kv, g * mq, dh)

    def cached(name):                                                      # [n, kv, keys, dh]
        x = st[name + "_pages"][st["table"].long()]
        if c["cache"] == "4bit":
            x = torch.stack((x & 15, x >> 4), 5).flatten(4).float().unflatten(4, (-1, GROUP))
            s = st[name + "_scale"][st["table"].long()].float()
            x = x.mul_(s[..., 0:1]).add_(s[..., 1:2]).flatten(4)
        return x.float().transpose(1, 2).flatten(2, 3)[:, :, :mk]

    s = torch.matmul(q, cached("k").transpose(2, 3)).view(n, kv, g, mq, mk).mul_(dh ** -0.5)
    j = torch.arange(mk, device=DEV)
    seen = j[None, None, :] < lk[:, None, None]
    if c["causal"]:       # the last query of a sequence sees all of its keys
        seen = seen & (j[None, None, :] <= i[None, :, None] + (lk - lq)[:, None, None])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(4, keepdim=True)
    o = torch.matmul(p.view(n, kv, g * mq, mk), cached("v")).view(n, kv, g, mq, dh) / total.clamp_min(1e-38)
    real = i[None, :] < lq[:, None]
    out = st["out"].clone()
    out[at[real]] = o.permute(0, 3, 1, 2, 4).reshape(n, mq, heads * dh)[real].to(out.dtype)
    if st["lse"] is None:
        return {"out": out}
    lse = st["lse"].clone()
    lse[at[real]] = (m + total.log()).squeeze(4).permute(0, 3, 1, 2).reshape(n, mq, heads)[real]
    return {"out": out, "lse": lse}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "linear8": _plain_linear8, "append": _plain_append, "paged": _plain_paged}


def _run_own(st):
    from paper_2510_03246_b200 import api
    c = st["case"]
    if c["kind"] == "norm":
        r = api.sp_rms_norm(st["X"], st["weight"], EPS, residual=st["R"], want_rstd=True,
                            out_dtype=torch.float8_e4m3fn if c["eight"] else None)
        out = {"rstd": r.rstd, "Y": r.Y}
        if st["R"] is not None:
            out["H"] = r.H
        if c["eight"]:
            out["scale"] = r.scale
        return out
    if c["kind"] == "norm_grad":
        dx, dw = api.sp_rms_norm_grad(st["dY"], st["H"], st["weight"], st["rstd"], d_stream=st["dH"])
        return {"dX": dx, "dweight": dw}
    if c["kind"] == "linear8":
        act = {"none": api.SP_LINEAR_NONE, "relu": api.SP_LINEAR_RELU, "silu": api.SP_LINEAR_SILU, "gelu": api.SP_LINEAR_GELU}[c["act"]]
        combine = api.SP_COMBINE_MUL if c["other"] == "mul" else api.SP_COMBINE_ADD
        return {"Y": api.sp_linear_e4m3(st["X"], st["X_scale"], st["W"], st["W_scale"], bias=st["bias"], act=act, other=st["other"],
                                        combine=combine)}
    pages = api.KvPages(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    if c["kind"] == "append":
        q, k = c["heads"] * c["dh"], c["kv"] * c["dh"]
        qkv = st["qkv"]
        turned = api.sp_cache_append(pages, qkv[:, q:q + k], qkv[:, q + k:], st["cu"], st["table"], st["lens"], Q=qkv[:, :q],
                                     inv_freq=st["inv_freq"], neighbours=c["pairs"] == "neighbours")
        K, V = api.sp_cache_read(pages, st["cu"], st["table"], st["lens"], qkv.shape[0], qkv.dtype)
        return {"Q": turned, "K": K, "V": V}
    out, lse = api.sp_cache_attention(st["Q"], pages, st["cu_q"], st["table"], st["lens"], c["heads"], causal=c["causal"],
                                      max_keys=st["keys"], out=st["out"], lse=st["lse"])
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def run(state):
    if own:
        return _run_own(state)
    return PLAIN[state["case"]["kind"]](state)


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n, T, d = case["T"] * case["d"], case["T"], case["d"]
        es, ss = (2 if case[k] == "bf16" else 4 for k in ("dtype", "stream"))
        more = ss if case["residual"] else 0
        if kind == "norm":
            return {"bytes": n * (es + 2 * more + (1 if case["eight"] else es)) + 4 * d + (8 if case["eight"] else 4) * T,
                    "flops": 5.0 * n}
        return {"bytes": n * (es + 2 * ss + more) + 8 * d + 4 * T, "flops": 10.0 * n}
    if kind == "linear8":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        return {"bytes": T * n_in + n_out * n_in + 4 * (T + n_out) + 2 * T * n_out * (2 if case["other"] != "none" else 1) +
                         (4 * n_out if case["bias"] else 0),
                "flops": 2.0 * T * n_in * n_out}
    heads, kv, dh = case["heads"], case["kv"], case["dh"]
    es = 2 if case["dtype"] == "bf16" else 4
    per_head = dh // 2 + 4 * (dh // GROUP) if case["cache"] == "4bit" else 2 * dh      # bytes of a token's key in the cache
    if kind == "append":
        T = sum(_lengths(case["new"]))
        # queries, keys and values read, turned queries and the cache written, the appended values read from it and written
        return {"bytes": T * (es * dh * (2 * heads + 4 * kv) + 4 * kv * per_head), "flops": 6.0 * T * (heads + kv) * dh}
    pairs = 0
    q_len, k_len = _lengths(case["q"]), _lengths(case["k"])
    for q, k in zip(q_len, k_len):
        pairs += q * k - q * (q - 1) // 2 if case["causal"] else q * k
    nq = sum(q_len)
    return {"bytes": es * dh * 2 * nq * heads + 2 * sum(k_len) * kv * per_head + (4 * nq * heads if case["lse"] else 0),
            "flops": 4.0 * pairs * heads * dh}


# --------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_turn(x, position, inv_freq, pairs):
    out = x.clone()
    n = inv_freq.numel()
    for i in range(n):
        a, b = (i, n + i) if pairs == "halves" else (2 * i, 2 * i + 1)
        angle = (position.double() * inv_freq[i].double())[:, None]
        out[..., a] = x[..., a] * torch.cos(angle) - x[..., b] * torch.sin(angle)
        out[..., b] = x[..., a] * torch.sin(angle) + x[..., b] * torch.cos(angle)
    return out


def _exact_cached(st, name, s, length):
    """[length, kv, dh] of sequence s."""
    c = st["case"]
    at = torch.arange(length, device=DEV)
    pg, slot = st["table"][s].long()[at // c["page"]], at % c["page"]
    x = st[name + "_pages"][pg, :, slot]
    if c["cache"] != "4bit":
        return x.double()
    full = torch.empty(length, c["kv"], c["dh"], dtype=torch.float64, device=DEV)
    full[..., 0::2], full[..., 1::2] = (x % 16).double(), (x // 16).double()
    s = st[name + "_scale"][pg, :, slot].double().repeat_interleave(GROUP, dim=2)
    return full * s[..., 0] + s[..., 1]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = st["X"].double() if st["R"] is None else st["X"].double() + st["R"].double()
        rms = torch.sqrt(torch.einsum("td,td->t", h, h) / case["d"] + EPS)
        y = h / rms[:, None] * st["weight"].double()
        out = {"rstd": 1 / rms, "Y": y}
        if st["R"] is not None:
            out["H"] = h
        if case["eight"]:
            out["scale"] = y.abs().max(dim=1).values / E4M3_MAX
            out["Y"] = y / out["scale"][:, None]
        return out
    if kind == "norm_grad":
        h, dy, r = st["H"].double(), st["dY"].double(), st["rstd"].double()
        wdy = dy * st["weight"].double()
        dx = wdy * r[:, None] - h * (r ** 3 * torch.einsum("td,td->t", wdy, h) / case["d"])[:, None]
        if st["dH"] is not None:
            dx = dx + st["dH"].double()
        return {"dX": dx, "dweight": torch.einsum("td,td,t->d", dy, h, r)}
    if kind == "linear8":
        y = torch.einsum("ti,oi->to", st["X"].double(), st["W"].double())
        y = y * st["X_scale"].double()[:, None] * st["W_scale"].double()[None, :]
        if case["bias"]:
            y += st["bias"].double()
        fn = {"none": lambda u: u, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
        y = fn[case["act"]](y)
        if case["other"] != "none":
            y = y + st["other"].double() if case["other"] == "add" else y * st["other"].double()
        return {"Y": y}
    heads, kv, dh = case["heads"], case["kv"], case["dh"]
    if kind == "append":
        q, k, v = heads * dh, kv * dh, kv * dh
        T = st["qkv"].shape[0]
        position = torch.cat([torch.arange(b, b + n, device=DEV) for n, b in zip(_lengths(case["new"]), _lengths(case["before"]))] or
                             [torch.zeros(0, device=DEV)])
        if position.numel() < T:
            return None
        Q, K, V = (x.double().view(T, -1, dh) for x in st["qkv"].split((q, k, v), 1))
        Q, K = (_exact_turn(x, position, st["inv_freq"], case["pairs"]) for x in (Q, K))
        if case["cache"] == "4bit":
            held = []
            for x in (K, V):
                x = x.reshape(T * kv * (dh // GROUP), GROUP)
                zero = x.min(dim=1, keepdim=True).values.to(torch.bfloat16).double()
                step = ((x.max(dim=1, keepdim=True).values - zero) / 15).to(torch.bfloat16).double()
                held.append((torch.clamp(torch.round((x - zero) / step.clamp_min(1e-300)), 0, 15) * step + zero).reshape(T, kv, dh))
            K, V = held
        return {"Q": Q.reshape(T, -1), "K": K.reshape(T, -1), "V": V.reshape(T, -1)}
    out = st["out"].double()
    lse = torch.zeros(out.shape[0], heads, dtype=torch.float64, device=DEV)
    cq, k_len = _offsets(_lengths(case["q"])), _lengths(case["k"])
    for s, nk in enumerate(k_len):
        rq, nq = slice(cq[s], cq[s + 1]), cq[s + 1] - cq[s]
        K, V = _exact_cached(st, "k", s, nk), _exact_cached(st, "v", s, nk)
        for h in range(heads):
            logits = st["Q"][rq, h * dh:(h + 1) * dh].double() @ K[:, h // (heads // kv)].T * dh ** -0.5
            if case["causal"]:
                logits[torch.ones(nq, nk, dtype=torch.bool, device=DEV).triu(nk - nq + 1)] = -math.inf
            lse[rq, h] = torch.logsumexp(logits, 1)
            out[rq, h * dh:(h + 1) * dh] = torch.softmax(logits, 1) @ V[:, h // (heads // kv)]
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
