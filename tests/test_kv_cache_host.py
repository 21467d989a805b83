"""The bookkeeping of pipeline.KvCache, on the host alone."""
import pytest
import torch

from paper_2510_03246_b200 import pipeline


def cache(n_pages=8, page_len=16, **kw):
    return pipeline.KvCache(2, n_pages, page_len, 1, 64, device="cpu", **kw)


def test_pages_of_a_text_grow_with_it():
    c = cache()
    s = c.step(["a", "b"], [17, 3])
    assert s.cu.tolist() == [0, 17, 20] and s.lens.tolist() == [17, 3] and s.fresh and s.keys == 20
    assert s.table.shape == (2, 2) and s.table[1, 1] == -1 and s.table.dtype == torch.int32
    used = set(s.table.flatten().tolist()) - {-1}
    assert len(used) == 3 and len(c) == 5
    t = c.step(["b", "a"], [13, 0])
    assert t.cu.tolist() == [0, 13, 13] and t.lens.tolist() == [16, 17] and not t.fresh and t.keys == 16
    assert t.table[0].tolist() == [int(s.table[1, 0]), -1] and t.table[1].tolist() == s.table[0].tolist() and len(c) == 5
    t = c.step(["b"], [1])
    assert t.lens.tolist() == [17] and t.table.shape == (1, 2) and len(c) == 4
    assert c.tokens("a") == 17 and c.tokens("b") == 17 and c.tokens("c") == 0


def test_freed_pages_are_used_again():
    c = cache(n_pages=4)
    c.step(["a"], [64])
    with pytest.raises(MemoryError):
        c.step(["b"], [1])
    assert c.tokens("b") == 0 and len(c) == 0
    c.close("a")
    c.close("a")
    c.close("never")
    assert len(c) == 4
    s = c.step(["b", "c"], [33, 16])
    assert sorted(set(s.table.flatten().tolist()) - {-1}) == [0, 1, 2, 3]


def test_what_does_not_fit_takes_nothing():
    c = cache(n_pages=3)
    c.step(["a"], [20])
    with pytest.raises(MemoryError):
        c.step(["a", "b"], [10, 20])
    assert c.tokens("a") == 20 and len(c) == 1
    assert c.step(["a"], [12]).lens.tolist() == [32] and len(c) == 1


def test_refusals():
    c = cache()
    for texts, new in ((["a", "a"], [1, 1]), (["a"], [1, 2]), (["a"], [-1])):
        with pytest.raises(ValueError):
            c.step(texts, new)
    assert len(c) == 8
    s = c.step([], [])
    assert s.cu.tolist() == [0] and s.keys == 0 and s.table.shape == (0, 0)
    s = c.step(["a"], [0])
    assert s.lens.tolist() == [0] and s.fresh and s.keys == 0


def test_layers_share_one_table_and_four_bits_have_scales():
    c = cache(four_bits=True)
    assert len(c.layers) == 2 and c.layers[0].k.shape == (8, 1, 16, 32) and c.layers[0].k_scale.shape == (8, 1, 16, 1, 2)
    assert c.layers[0].k.dtype == torch.uint8 and c.layers[1].v_scale.dtype == torch.bfloat16


def test_weights_in_8_bits():
    W = torch.randn(5, 37)
    W[3] = 0
    W8, scale = pipeline.weights_8bit(W)
    assert W8.dtype == torch.float8_e4m3fn and W8.stride(0) % 16 == 0 and scale.dtype == torch.float32
    back = W8.float() * scale[:, None]
    assert ((back - W).abs() <= W.abs() * 2.0 ** -4 + scale[:, None] * 2.0 ** -10 + 1e-7 * W.abs()).all()


def test_projections_of_other_heads_are_refused():
    cache = pipeline.KvCache(1, 4, 16, 2, 64, device="cpu")
    step = cache.step(["a"], [3])
    for heads, kv, cols in ((4, 2, 8 * 64 + 16), (4, 2, 7 * 64), (8, 2, 8 * 64)):
        with pytest.raises(ValueError, match="columns"):
            pipeline.cached_attention(torch.zeros(3, cols), cache.layers[0], step, heads, kv)
