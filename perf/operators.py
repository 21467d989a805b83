"""The operators that carry activations through a (pruned) layer and score a model's predictions, as cases of one call each.

  attention  causal attention over packed sequences with grouped heads: the head outputs of a calibration set or of a text
             to be scored, from one token after a long cache to whole prompts
  linear     a projection with what follows it in a layer: bias, activation, then the residual added or the other branch
             of a gated module multiplied
  loss       log probability of given tokens with the entropy of each row and its best alternatives
  loss_grad  the gradient of those log probabilities and entropies with respect to the logits

Head layouts and widths are those of the repository's workloads (12 x 64, 32 x 64, 32 x 128 heads; widths 768 to 4096, FFN
widths cut by its sparsities, so that kept counts are odd), grouped key and value heads and vocabularies are generic.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attn(name, q, k, heads, kv, dh, **kw):
    q, k = (" ".join(map(str, x)) for x in (q, k))          # lengths of the sequences: queries, keys
    c = dict(name=name, kind="attention", q=q, k=k, heads=heads, kv=kv, dh=dh, dtype="bf16", causal=True, tail=0, lse=True)
    c.update(kw)
    return c


def _lin(name, T, n_in, n_out, **kw):
    c = dict(name=name, kind="linear", T=T, n_in=n_in, n_out=n_out, dtype="bf16", bias=True, act="none", other="none")
    c.update(kw)
    return c


def _loss(name, kind, T, V, **kw):
    c = dict(name=name, kind=kind, T=T, V=V, dtype="bf16", alts=0, entropy=True, scale=1.0, ignored=0.05)
    c.update(kw)
    return c


def listed():
    return [
        # one new token against a short cache, the smallest model's heads: latency alone
        _attn("attn_token_768", [1], [777], 12, 12, 64),
        # a batch of single tokens, caches of many lengths: bound by reading the caches
        _attn("attn_tokens_long", [1] * 16, [2048 + 1931 * i for i in range(16)], 32, 8, 128),
        # 16 calibration segments of 128 tokens in fp32 storage, the smallest model's heads
        _attn("attn_segments_f32", [128] * 16, [128] * 16, 12, 12, 64, dtype="f32"),
        # packed documents of very different lengths in one row of tokens, grouped heads, a padded end
        _attn("attn_documents", [2048, 1, 977, 130, 1500, 64, 2047, 333, 19, 1216, 700, 2, 1801, 255, 512, 1111],
              [2048, 1, 977, 130, 1500, 64, 2047, 333, 19, 1216, 700, 2, 1801, 255, 512, 1111], 32, 8, 64, tail=83),
        # one long prompt, 32 heads of 128 on 8 key and value heads: bound by the matrix products
        _attn("attn_prompt_8192", [8192], [8192], 32, 8, 128),
        # the up projection of the smallest model on a few tokens: bound by reading the weight once
        _lin("linear_768_few", 16, 768, 1536, act="relu"),
        # the down projection of a layer pruned to an odd number of channels, residual added, a chunk of tokens
        _lin("linear_down_6554", 8192, 6554, 4096, other="add"),
        # gate branch of a gated module pruned to 30 %: silu of the product times the up branch
        _lin("linear_gate_3303", 16384, 4096, 3303, bias=False, act="silu", other="mul"),
        # one prediction with its five best alternatives
        _loss("loss_1x32000", "loss", 1, 32000, dtype="f32", alts=5),
        # the tokens of four segments of 2048 scored at once, an odd vocabulary: bound by reading the logits once
        _loss("loss_8192x50257", "loss", 8192, 50257, alts=8),
        # gradient for a short batch in fp32
        _loss("loss_grad_100x50257", "loss_grad", 100, 50257, dtype="f32", entropy=False),
        # gradient of log probability and entropy over a large vocabulary: bound by reading and writing the logits
        _loss("loss_grad_4096x128256", "loss_grad", 4096, 128256, scale=0.7),
    ]


def _lengths(text):
    return [int(x) for x in text.split()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "linear", "loss", "loss_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "attention":
        dh = rng.choice([64, 128, 64, 128, 80, 96, 40])
        kv = rng.choice([1, 2, 4, 8, 12])
        heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
        form = rng.choice(["tokens", "packed", "chunk", "full"])
        if form == "tokens":                      # single tokens after caches of any length
            n = _log_int(rng, 1, 64)
            q, k = [1] * n, [_log_int(rng, 1, 32768) for _ in range(n)]
        elif form == "chunk":                     # the next tokens of a text of which a part is there already
            n = _log_int(rng, 1, 4)
            q = [_log_int(rng, 1, 700) for _ in range(n)]
            k = [x + _log_int(rng, 1, 6000) for x in q]
        else:
            n = _log_int(rng, 1, 12)
            q = [_log_int(rng, 1, 2048) for _ in range(n)]
            k = list(q)
        while len(q) > 1 and len(q) * heads * max(q) * max(k) > 1 << 30:
            q, k = q[:-1], k[:-1]
        return _attn(None, q, k, heads, kv, dh, dtype=dtype, causal=form != "full", tail=rng.choice([0, 0, 1, 17]),
                     lse=rng.random() < 0.7)
    if kind == "linear":
        n_in, n_out = (_log_int(rng, 64, 6000) for _ in range(2))
        top = (2 * 8192 * 6554 * 4096) // (2 * n_in * n_out)
        T = _log_int(rng, 1, min(16384 if dtype == "bf16" else 4096, max(1, top)))
        return _lin(None, T, n_in, n_out, dtype=dtype, bias=rng.random() < 0.6,
                    act=rng.choice(["none", "relu", "silu", "gelu"]), other=rng.choice(["none", "add", "mul"]))
    V = _log_int(rng, 1000, 131072)
    T = _log_int(rng, 1, min(8192, (256 << 20) // V))
    return _loss(None, kind, T, V, dtype=dtype, alts=rng.choice([0, 1, 5, 20]), entropy=rng.random() < 0.6,
                 scale=rng.choice([1.0, 0.7, 1.6]), ignored=rng.choice([0.0, 0.05, 0.5]))


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _wide(rows, cols, dtype):
    """[rows, cols] whose rows start on 16 bytes, as a program lays out activations of an odd width."""
    return torch.zeros(rows, (cols + 7) // 8 * 8, dtype=dtype, device=DEV)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    st = {"case": case}
    if case["kind"] == "attention":
        heads, kv, dh = case["heads"], case["kv"], case["dh"]
        cq, ck = _offsets(_lengths(case["q"])), _offsets(_lengths(case["k"]))
        nq, nk = cq[-1] + case["tail"], ck[-1] + case["tail"]
        # a few strong channels in queries and keys, so that rows differ in how peaked they are
        strong = 1.0 + 3.0 * (torch.rand(dh, generator=g, device=DEV) < 0.03)
        st["Q"] = (normal(nq, heads, dh) * strong).reshape(nq, heads * dh).to(dt)
        st["K"] = normal(nk, kv * dh).to(dt)
        st["V"] = normal(nk, kv * dh).to(dt)
        st["cu_q"] = torch.tensor(cq, dtype=torch.int32, device=DEV)
        st["cu_k"] = torch.tensor(ck, dtype=torch.int32, device=DEV)
        st["out"] = torch.zeros(nq, heads * dh, dtype=dt, device=DEV)        # the caller's buffers: rows behind the last
        st["lse"] = torch.zeros(nq, heads, device=DEV) if case["lse"] else None    # sequence stay as they are
        return st
    if case["kind"] == "linear":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        x = _wide(T, n_in, dt)
        strong = 1.0 + 29.0 * (torch.rand(n_in, generator=g, device=DEV) < 0.005)    # outlier channels of calibration inputs
        x.copy_(normal(T, n_in) * strong)
        w = _wide(n_out, n_in, dt)
        w.copy_(normal(n_out, n_in) / math.sqrt(n_in))
        st["X"], st["W"] = x, w
        st["bias"] = 0.1 * normal(n_out) if case["bias"] else None
        st["other"] = None
        if case["other"] != "none":
            st["other"] = _wide(T, n_out, dt)
            st["other"].copy_(normal(T, n_out))
        return st
    T, V = case["T"], case["V"]
    x = torch.empty(T, V, dtype=dt, device=DEV)
    for t in range(0, T, 1024):                   # logits as a model leaves them: most near zero, some tokens far above
        part = normal(min(1024, T - t), V)
        x[t:t + 1024] = part * (1.5 + part.relu())
    st["logits"] = x
    target = torch.randint(0, V, (T,), generator=g, device=DEV)
    target[torch.rand(T, generator=g, device=DEV) < case["ignored"]] = -100
    st["targets"] = target
    if case["kind"] == "loss_grad":
        st["g_logp"] = normal(T)
        st["g_entropy"] = normal(T) if case["entropy"] else None
        st["lse"] = torch.cat([torch.logsumexp(x[t:t + 1024].double() * case["scale"], 1) for t in range(0, T, 1024)]).float()
        st["entropy"] = None
        if case["entropy"]:
            parts = []
            for t in range(0, T, 1024):
                z = torch.log_softmax(x[t:t + 1024].double() * case["scale"], 1)
                parts.append(-(z.exp() * z).sum(1))
            st["entropy"] = torch.cat(parts).float()
    return st


# ------------------------------------------------------------------------------------------------- plain forms, 32 bits
def _padded(x, cu, lengths, width, heads, dh):
    """[n_seq, width, heads, dh] of packed rows; rows beyond a sequence repeat some row and are masked by the caller."""
    at = (cu[:-1, None].long() + torch.arange(width, device=DEV)[None, :]).clamp(max=x.shape[0] - 1)
    return x.float().view(x.shape[0], heads, dh)[at], at, torch.arange(width, device=DEV)[None, :] < lengths[:, None]


def _plain_attention(st):
    c = st["case"]
    heads, kv, dh = c["heads"], c["kv"], c["dh"]
    q_len, k_len = _lengths(c["q"]), _lengths(c["k"])
    n, g, mq, mk = len(q_len), heads // kv, max(q_len), max(k_len)
    lq, lk = st["cu_q"][1:] - st["cu_q"][:-1], st["cu_k"][1:] - st["cu_k"][:-1]
    q, at, real_q = _padded(st["Q"], st["cu_q"], lq, mq, heads, dh)
    k, _, real_k = _padded(st["K"], st["cu_k"], lk, mk, kv, dh)
    v, _, _ = _padded(st["V"], st["cu_k"], lk, mk, kv, dh)
    q = q.view(n, mq, kv, g, dh).permute(0, 2, 3, 1, 4).reshape(n, kv, g * mq, dh)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).view(n, kv, g, mq, mk).mul_(1.0 / math.sqrt(dh))
    seen = real_k[:, None, :]
    if c["causal"]:       # the last query of a sequence sees all of its keys
        i = torch.arange(mq, device=DEV)[None, :, None] + (lk - lq)[:, None, None]
        seen = seen & (torch.arange(mk, device=DEV)[None, None, :] <= i)
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(4, keepdim=True)
    o = torch.matmul(p.view(n, kv, g * mq, mk), v.permute(0, 2, 1, 3)).view(n, kv, g, mq, dh) / total.clamp_min(1e-38)
    out = st["out"].clone()
    rows = at[real_q]
    out[rows] = o.permute(0, 3, 1, 2, 4).reshape(n, mq, heads * dh)[real_q].to(out.dtype)
    if st["lse"] is None:
        return {"out": out}
    lse = st["lse"].clone()
    lse[rows] = (m + total.log()).squeeze(4).permute(0, 3, 1, 2).reshape(n, mq, heads)[real_q]
    return {"out": out, "lse": lse}


def _activate(y, act):
    if act == "relu":
        return y.clamp_min(0)
    if act == "silu":
        return y / (1 + (-y).exp())
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain_linear(st):
    c = st["case"]
    y = torch.matmul(st["X"].float(), st["W"].float().t())
    if st["bias"] is not None:
        y = y + st["bias"]
    y = _activate(y, c["act"])
    if c["other"] == "add":
        y = y + st["other"].float()
    elif c["other"] == "mul":
        y = y * st["other"].float()
    return {"Y": y.to(st["X"].dtype)}


def _plain_loss(st):
    c = st["case"]
    z = st["logits"].float() * c["scale"]
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1)
    lse = m.squeeze(1) + total.log()
    t = st["targets"]
    logp = torch.where(t < 0, torch.zeros_like(lse), z.gather(1, t.clamp_min(0)[:, None]).squeeze(1) - lse)
    out = {"logp": logp, "lse": lse}
    if c["entropy"]:
        out["entropy"] = total.log() - (e * (z - m)).sum(1) / total
    if c["alts"]:
        # whole keys that order as (value, then the lower index): no two are equal
        b = (st["logits"].float() + 0.0).view(torch.int32).long()
        key = torch.where(b >= 0, b, b ^ 0x7FFFFFFF) * (1 << 32) + (0x7FFFFFFF - torch.arange(z.shape[1], device=DEV))
        ids = 0x7FFFFFFF - (torch.topk(key, c["alts"], dim=1).values & 0xFFFFFFFF)
        out["alt_ids"] = ids.int()
        out["alt_logp"] = z.gather(1, ids) - lse[:, None]
    return out


def _plain_loss_grad(st):
    c = st["case"]
    z = st["logits"].float() * c["scale"]
    logp = z - st["lse"][:, None]
    p = logp.exp()
    t = st["targets"]
    gl = torch.where(t < 0, torch.zeros_like(st["g_logp"]), st["g_logp"])
    d = p * -gl[:, None]
    if c["entropy"]:
        d = d - st["g_entropy"][:, None] * p * (logp + st["entropy"][:, None])
    d.scatter_add_(1, t.clamp_min(0)[:, None], gl[:, None])
    return {"dlogits": (d * c["scale"]).to(st["logits"].dtype)}


PLAIN = {"attention": _plain_attention, "linear": _plain_linear, "loss": _plain_loss, "loss_grad": _plain_loss_grad}


def _run_own(st):
    from paper_2510_03246_b200 import api
    c = st["case"]
    if c["kind"] == "attention":
        out, lse = api.sp_attention(st["Q"], st["K"], st["V"], st["cu_q"], st["cu_k"], c["heads"], c["kv"],
                                    causal=c["causal"], out=st["out"], lse=st["lse"])
        return {"out": out, "lse": lse} if c["lse"] else {"out": out}
    if c["kind"] == "linear":
        act = {"none": api.SP_LINEAR_NONE, "relu": api.SP_LINEAR_RELU, "silu": api.SP_LINEAR_SILU,
               "gelu": api.SP_LINEAR_GELU}[c["act"]]
        combine = api.SP_COMBINE_MUL if c["other"] == "mul" else api.SP_COMBINE_ADD
        return {"Y": api.sp_linear(st["X"], st["W"], bias=st["bias"], act=act, other=st["other"], combine=combine)}
    if c["kind"] == "loss":
        r = api.sp_token_logprobs(st["logits"], st["targets"], n_alts=c["alts"], scale=c["scale"],
                                  want_entropy=c["entropy"])
        out = {"logp": r.logp, "lse": r.lse}
        if c["entropy"]:
            out["entropy"] = r.entropy
        if c["alts"]:
            out["alt_ids"], out["alt_logp"] = r.alt_ids, r.alt_logp
        return out
    return {"dlogits": api.sp_token_logprobs_grad(st["logits"], st["targets"], st["lse"], st["g_logp"],
                                                  entropy=st["entropy"], g_entropy=st["g_entropy"], scale=c["scale"])}


def run(state):
    if own:
        return _run_own(state)
    return PLAIN[state["case"]["kind"]](state)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "attention":
        heads, kv, dh = case["heads"], case["kv"], case["dh"]
        pairs = 0
        q_len, k_len = _lengths(case["q"]), _lengths(case["k"])
        for q, k in zip(q_len, k_len):
            pairs += q * k - q * (q - 1) // 2 if case["causal"] else q * k
        nq, nk = sum(q_len), sum(k_len)
        return {"bytes": es * dh * (2 * nq * heads + 2 * nk * kv) + (4 * nq * heads if case["lse"] else 0),
                "flops": 4.0 * pairs * heads * dh}
    if case["kind"] == "linear":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        return {"bytes": es * (T * n_in + n_out * n_in + T * n_out * (2 if case["other"] != "none" else 1)) +
                         (4 * n_out if case["bias"] else 0),
                "flops": 2.0 * T * n_in * n_out}
    T, V = case["T"], case["V"]
    if case["kind"] == "loss":
        return {"bytes": es * T * V + T * (8 + 8 + (4 if case["entropy"] else 0) + 8 * case["alts"]),
                "flops": float(T) * V * (6 if case["entropy"] else 4)}
    return {"bytes": 2 * es * T * V + T * (16 + (8 if case["entropy"] else 0)),
            "flops": float(T) * V * (8 if case["entropy"] else 5)}


# --------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attention":
        heads, kv, dh = case["heads"], case["kv"], case["dh"]
        out = st["out"].double()
        lse = torch.zeros(out.shape[0], heads, dtype=torch.float64, device=DEV)
        cq, ck = _offsets(_lengths(case["q"])), _offsets(_lengths(case["k"]))
        for s in range(len(cq) - 1):
            rq, rk = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s + 1])
            nq, nk = cq[s + 1] - cq[s], ck[s + 1] - ck[s]
            for h in range(heads):
                j = h // (heads // kv)
                logits = st["Q"][rq, h * dh:(h + 1) * dh].double() @ st["K"][rk, j * dh:(j + 1) * dh].double().T
                logits = logits * dh ** -0.5
                if case["causal"]:
                    hidden = torch.ones(nq, nk, dtype=torch.bool, device=DEV).triu(nk - nq + 1)
                    logits[hidden] = -math.inf
                lse[rq, h] = torch.logsumexp(logits, 1)
                out[rq, h * dh:(h + 1) * dh] = torch.softmax(logits, 1) @ st["V"][rk, j * dh:(j + 1) * dh].double()
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    if case["kind"] == "linear":
        y = torch.einsum("ti,oi->to", st["X"].double(), st["W"].double())
        if case["bias"]:
            y += st["bias"].double()
        fn = {"none": lambda u: u, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
        y = fn[case["act"]](y)
        if case["other"] != "none":
            y = y + st["other"].double() if case["other"] == "add" else y * st["other"].double()
        return {"Y": y}
    parts = []
    for t in range(0, case["T"], 512):
        x = st["logits"][t:t + 512].double()
        lp = torch.log_softmax(x * case["scale"], 1)
        tg = st["targets"][t:t + 512]
        rows = torch.arange(len(tg), device=DEV)
        told = tg >= 0
        if case["kind"] == "loss":
            r = {"logp": torch.where(told, lp[rows, tg.clamp_min(0)], 0.0), "lse": torch.logsumexp(x * case["scale"], 1)}
            if case["entropy"]:
                r["entropy"] = torch.special.entr(lp.exp()).sum(1)
            if case["alts"]:
                ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["alts"]]
                r["alt_ids"], r["alt_logp"] = ids.int(), lp.gather(1, ids)
        else:
            d = -lp.exp()
            d[rows[told], tg[told]] += 1
            d *= torch.where(told, st["g_logp"][t:t + 512].double(), 0.0)[:, None]
            if case["entropy"]:
                h = -(lp.exp() * lp).sum(1, keepdim=True)
                d -= st["g_entropy"][t:t + 512].double()[:, None] * lp.exp() * (lp + h)
            r = {"dlogits": d * case["scale"]}
        parts.append(r)
    return {key: torch.cat([r[key] for r in parts]) for key in parts[0]}
