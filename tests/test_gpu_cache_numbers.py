"""The 4-bit numbers that sp_cache_append writes are those of the formula in 64 bits, bit for bit, wherever rounding could go either way."""
import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def formula(x):
    """x [N, kv, groups, 64] in 64 bits -> numbers, zero, scale (rounded to fp32 and from there to bf16), and which groups are finite."""
    fine = x.float().isfinite().all(3)
    x = torch.where(fine[..., None], x, torch.zeros_like(x))
    zero = x.amin(3).float().bfloat16()
    scale = ((x.amax(3) - zero.double()) / 15.0).float().bfloat16()
    s = scale.double()
    n = ((x - zero.double()[..., None]) / torch.where(s > 0, s, torch.ones_like(s))[..., None]).round().clamp(0, 15)
    return torch.where((s > 0)[..., None], n, torch.zeros_like(n)).to(torch.uint8), zero, scale, fine


def check(pages, which, want, table, n, page):
    n_want, zero, scale, fine = formula(want)
    data, pair = (pages.k, pages.k_scale) if which == "k" else (pages.v, pages.v_scale)
    rows = torch.arange(n, device=DEV)
    pg, slot = table[0, rows // page].long(), rows % page
    b = data[pg, :, slot]                                        # [n, kv, dh / 2]
    got = torch.stack([b & 15, b >> 4], 3).flatten(2).view(n_want.shape)
    z, s = pair[pg, :, slot][..., 1], pair[pg, :, slot][..., 0]
    assert z[~fine].isnan().all()
    assert torch.equal(got[fine], n_want[fine])
    assert torch.equal(z[fine], zero[fine]) and torch.equal(s[fine], scale[fine])


def values(kind, n, kv, dh, g):
    x = torch.randn(n, kv * dh, generator=g, device=DEV)
    if kind == "steps":                                          # borders of two steps everywhere
        x = torch.randint(-128, 128, x.shape, generator=g, device=DEV) / 16.0
    elif kind == "ladder":                                       # halves of the step itself, which is 1
        x = torch.randint(0, 31, x.shape, generator=g, device=DEV) / 2.0
        x.view(n, kv, -1, 64)[..., 0] = 0.0
        x.view(n, kv, -1, 64)[..., 1] = 15.0
    elif kind == "wide":
        x = x * 2.0 ** torch.randint(-30, 30, x.shape, generator=g, device=DEV)
    elif kind == "offset":                                       # far from zero: few steps apart
        x = x + 1000.0
    elif kind == "equal":
        x = x[:, :1].expand(n, kv * dh).contiguous()
    elif kind == "tiny":
        x = x * 1e-37
    elif kind == "huge":
        x = x.sign() * 1e38 * (1 + x.abs())
    elif kind == "odd":
        x[::3, 5] = float("nan")
        x[1::3, dh - 1] = float("inf")
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["normal", "steps", "ladder", "wide", "offset", "equal", "tiny", "huge", "odd"])
def test_numbers_of_given_values(kind, dtype):
    n, kv, dh, page = 700, 3, 128, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    K, V = (values(kind, n, kv, dh, g).to(dtype) for _ in range(2))
    pages = api.KvPages.empty(11, kv, page, dh, True)
    table = torch.randperm(11, generator=torch.Generator().manual_seed(1))[None].int().to(DEV)
    api.sp_cache_append(pages, K, V, torch.tensor([0, n], dtype=torch.int32, device=DEV), table, torch.tensor([n], dtype=torch.int32, device=DEV))
    for which, x in (("k", K), ("v", V)):
        check(pages, which, x.double().view(n, kv, dh // 64, 64), table, n, page)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("kind", ["normal", "steps", "far"])
@pytest.mark.parametrize("dh, turned", [(64, 64), (128, 128), (128, 32)])
def test_numbers_of_turned_keys(dh, turned, kind, neighbours):
    """`far`: partners 2^14 times as large as the group's own values.  (Cosines of the two sides may differ in the last of 53 bits: a value would have
    to lie within 2^-50 of a border for that to show; position 0 turns by an angle of 0, whose borders are exact.)"""
    n, kv, page = 900, 2, 16
    g = torch.Generator(device=DEV).manual_seed(5)
    K = values("normal" if kind == "far" else kind, n, kv, dh, g)
    if kind == "far":
        K.view(n, kv, 2, dh // 2)[:, :, 1] *= 2.0 ** 14
    K = K.bfloat16()
    f = 10000.0 ** (-2.0 * torch.arange(turned // 2, device=DEV).float() / turned)
    pages = api.KvPages.empty(57, kv, page, dh, True)
    table = torch.randperm(57, generator=torch.Generator().manual_seed(2))[None].int().to(DEV)
    position = torch.randint(0, 100000, (n,), generator=g, device=DEV).int()
    position[::4] = 0
    api.sp_cache_append(pages, K, K, torch.tensor([0, n], dtype=torch.int32, device=DEV), table, torch.tensor([n], dtype=torch.int32, device=DEV),
                        inv_freq=f, neighbours=neighbours, positions=position)
    x = K.double().view(n, kv, dh).clone()
    at, bt = (slice(0, turned, 2), slice(1, turned, 2)) if neighbours else (slice(0, turned // 2), slice(turned // 2, turned))
    angle = position.double()[:, None, None] * f.double()
    a, b, c, s = x[..., at].clone(), x[..., bt].clone(), angle.cos(), angle.sin()
    x[..., at], x[..., bt] = a * c - b * s, b * c + a * s
    check(pages, "k", x.view(n, kv, dh // 64, 64), table, n, page)
