"""sp_linear_e4m3 against its formula in 64 bits.  Products of two 8-bit values are exact in fp32; a sum over K of them in fp32 is off by at most K
roundings of 2^-24 of the sum of magnitudes (in the matrix units, which add a group of products at a time and may cut instead of round, 2^-23 for
every 16), the result by half a step more; the activations by 2^-16 of the value."""
import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8, BF, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32
ACTS = {api.SP_LINEAR_NONE: lambda u: u, api.SP_LINEAR_RELU: torch.relu, api.SP_LINEAR_SILU: torch.nn.functional.silu,
        api.SP_LINEAR_GELU: torch.nn.functional.gelu}


def eight(rows, cols, seed, pad=0):
    """[rows, cols] of e4m3 whose rows start on 16 bytes, scales; what stands behind a row's last value is NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    full = torch.randn(rows, cols, generator=g, device=DEV)
    scale = full.abs().amax(1) / 448
    wide = (cols + 15) // 16 * 16 + pad
    buf = torch.full((rows, wide), 127, dtype=torch.uint8, device=DEV).view(F8)
    buf[:, :cols] = (full / scale[:, None]).clamp(-448, 448).to(F8)
    return buf[:, :cols], scale


def check(X, xs, W, ws, Y, bias=None, act=api.SP_LINEAR_NONE, other=None, combine=api.SP_COMBINE_ADD):
    K = X.shape[1]
    size = (X.double().abs() @ W.double().abs().t()) * xs.double()[:, None] * ws.double()
    y = (X.double() @ W.double().t()) * xs.double()[:, None] * ws.double()
    off = size * (K / 16 + 4) * 2.0 ** -23
    if bias is not None:
        y = y + bias.double()
        off = off + 2.0 ** -24 * y.abs()
    y = ACTS[act](y)
    off = 1.2 * off + 2.0 ** -16 * y.abs()                       # (no activation is steeper than 1.13)
    if other is not None:
        if combine == api.SP_COMBINE_ADD:
            y, off = y + other.double(), off
        else:
            y, off = y * other.double(), off * other.double().abs()
    half = 2.0 ** -8 if Y.dtype == BF else 2.0 ** -24
    assert ((Y.double() - y).abs() <= off + half * y.abs() + 1e-30).all()


@pytest.mark.parametrize("T, K, N", [(1, 1, 1), (1, 64, 64), (3, 17, 5), (8, 768, 1536), (16, 4096, 33), (17, 100, 4097), (40, 513, 1000),
                                     (64, 4096, 4096), (192, 127, 1365), (193, 128, 2048), (256, 129, 256), (300, 4000, 301),
                                     (1000, 2048, 7), (1025, 65, 9), (2048, 1000, 3303)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_sizes(T, K, N, dtype):
    X, xs = eight(T, K, 1)
    W, ws = eight(N, K, 2, pad=16)
    Y = api.sp_linear_e4m3(X, xs, W, ws, out_dtype=dtype)
    assert Y.dtype == dtype
    check(X, xs, W, ws, Y)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("combine", [None, api.SP_COMBINE_ADD, api.SP_COMBINE_MUL])
@pytest.mark.parametrize("T, N", [(5, 500), (700, 500), (700, 501)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_epilogues(act, combine, T, N, dtype):
    X, xs = eight(T, 400, 3)
    W, ws = eight(N, 400, 4)
    bias = torch.randn(N, device=DEV)
    other = None if combine is None else api.rows_of_16_bytes(T, N, dtype, DEV)
    kw = {}
    if other is not None:
        other.copy_(torch.randn(T, N, device=DEV))
        kw = dict(other=other, combine=combine)
    Y = api.sp_linear_e4m3(X, xs, W, ws, bias=bias, act=act, out_dtype=dtype, **kw)
    check(X, xs, W, ws, Y, bias=bias, act=act, **kw)
    if other is not None:                                        # in the place of `other`
        place = other.clone(memory_format=torch.preserve_format) if other.is_contiguous() else None
        if place is not None:
            assert torch.equal(api.sp_linear_e4m3(X, xs, W, ws, bias=bias, act=act, other=place, combine=combine, out=place), Y)


@pytest.mark.parametrize("T", [4, 300])
def test_unaligned_results_and_their_surroundings(T):
    X, xs = eight(T, 96, 5)
    W, ws = eight(75, 96, 6)
    for dtype in (BF, F32):
        buf = torch.full((T + 2, 83), 7.0, dtype=dtype, device=DEV)
        out = buf[1:-1, 3:78]
        check(X, xs, W, ws, api.sp_linear_e4m3(X, xs, W, ws, out=out))
        assert (buf[0] == 7).all() and (buf[-1] == 7).all() and (buf[:, :3] == 7).all() and (buf[:, 78:] == 7).all()


@pytest.mark.parametrize("T", [1, 16, 512])
def test_sums_keep_their_small_terms(T):
    """448 * 448 and then ones: all partial sums are whole numbers below 2^24, exact in fp32 in any order and grouping."""
    K = 8192
    x = torch.ones(T, K, device=DEV)
    x[:, 0] = 448
    w = torch.ones(40, K, device=DEV)
    w[:, 0] = 448
    one = lambda n: torch.ones(n, device=DEV)
    Y = api.sp_linear_e4m3(x.to(F8), one(T), w.to(F8), one(40), out_dtype=F32)
    assert (Y == 448.0 * 448.0 + K - 1).all()
    x[:, 0] = 0
    x[:, 1::2] = 2.0 ** -9                                       # the smallest value
    Y = api.sp_linear_e4m3(x.to(F8), one(T), w.to(F8), one(40), out_dtype=F32)
    assert (Y == K // 2 - 1 + K // 2 * 2.0 ** -9).all()


def test_nan_stays_in_its_row_and_output():
    for T in (9, 300):
        X, xs = eight(T, 200, 7)
        W, ws = eight(64, 200, 8)
        X.view(torch.uint8)[4, 199] = 127
        W.view(torch.uint8)[11, 0] = 127
        Y = api.sp_linear_e4m3(X, xs, W, ws, out_dtype=F32)
        bad = torch.zeros(T, 64, dtype=torch.bool, device=DEV)
        bad[4] = True
        bad[:, 11] = True
        assert torch.equal(Y.isnan(), bad)
