"""What the prompt of a new text reads in pipeline.cached_attention: by itself its own keys and values, beside a text that goes on what the pages hold,
and a text without new tokens changes neither."""
import pytest
import torch

from paper_2510_03246_b200 import api, pipeline

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32 = torch.float32


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("beside", ["nothing", "no new tokens", "a token"])
def test_a_prompt_beside_a_running_text(beside, four):
    heads, kv, dh, n = 4, 2, 64, 70
    g = torch.Generator(device=DEV).manual_seed(5)
    cache = pipeline.KvCache(1, 64, 16, kv, dh, four)
    width = (heads + 2 * kv) * dh
    pipeline.cached_attention(torch.randn(100, width, generator=g, device=DEV), cache.layers[0], cache.step(["a"], [100]), heads, kv)
    prompt = torch.randn(n, width, generator=g, device=DEV)
    texts, new = {"nothing": (["p"], [n]), "no new tokens": (["p", "a"], [n, 0]), "a token": (["p", "a"], [n, 1])}[beside]
    x = torch.cat((prompt, torch.randn(1, width, generator=g, device=DEV))) if beside == "a token" else prompt
    step = cache.step(texts, new)
    assert step.fresh == (beside != "a token")
    H = pipeline.cached_attention(x.clone(), cache.layers[0], step, heads, kv)[:n]
    q, k, v = prompt[:, :heads * dh], prompt[:, heads * dh:(heads + kv) * dh], prompt[:, (heads + kv) * dh:]
    if not step.fresh:
        k, v = api.sp_cache_read(cache.layers[0], step.cu[:2].contiguous(), step.table[:1], step.lens[:1], n, F32)
    q, k, v = (t.double().view(n, -1, dh) for t in (q, k, v))
    z = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(heads // kv, 1)) * dh ** -0.5
    z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -torch.inf)
    want = torch.einsum("hij,jhd->ihd", torch.softmax(z, 2), v.repeat_interleave(heads // kv, 1)).flatten(1)
    # fp32 throughout: sums of 64 products and of at most 70 weights, 2^-18 of their terms' sizes (below 2^5 in the logits)
    assert (H.double() - want).abs().max() <= (2.0 ** -18 * 32 * 2 + 2.0 ** -18) * v.abs().max()
