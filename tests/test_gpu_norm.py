"""sp_rms_norm and sp_rms_norm_grad against their formulas in 64 bits.

Tolerances count roundings: half a step of the result's type (bf16 2^-8, fp32 2^-24, e4m3 2^-4 of the value, 2^-10 of the scale below its
normal range), and for sums in fp32 the number of additions that one value passes through (eight of a chunk, four chunks, five of a warp, 32 warps; a
512th of a row in the looping form) times 2^-24 of the sum of magnitudes."""
import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def rows(T, d, dtype, pad=0, shift=0, seed=0, scale=1.0):
    """[T, d] with `pad` more columns to a row, `shift` values into its buffer."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.randn(T * (d + pad) + shift, generator=g, device=DEV).mul_(scale).to(dtype)
    return buf[shift:].as_strided((T, d), (d + pad, 1))


def additions(d):
    return 64 + d / 512


def check_norm(X, R, w, eps, r, eight):
    h = X.double() + (R.double() if R is not None else 0.0)
    d = X.shape[1]
    rstd = (h.square().mean(1) + eps).rsqrt()
    assert ((r.rstd.double() - rstd).abs() <= rstd * additions(d) * 2.0 ** -24).all()
    y = h * rstd[:, None] * (w.double() if w is not None else 1.0)
    near = y.abs() * additions(d) * 2.0 ** -24
    if R is not None:
        assert ((r.H.double() - h).abs() <= h.abs() * HALF[R.dtype] + 2.0 ** -24 * (X.double().abs() + R.double().abs())).all()
    if eight:
        top = y.abs().amax(1).clamp_min(1e-30)
        assert ((r.scale.double() * 448 - top).abs() <= top * additions(d) * 2.0 ** -24).all()
        back = r.Y.double() * r.scale.double()[:, None]
        assert ((back - y).abs() <= y.abs() * 2.0 ** -4 + r.scale.double()[:, None] * 2.0 ** -10 + 2 * near).all()
    else:
        assert r.Y.dtype == X.dtype
        assert ((r.Y.double() - y).abs() <= y.abs() * HALF[X.dtype] + near + 1e-40).all()


@pytest.mark.parametrize("d", [1, 7, 8, 64, 333, 768, 1024, 1032, 4095, 4096, 5000, 8192, 8200, 32768, 33000])
@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("dx, dr", [(BF, BF), (BF, F32), (F32, F32), (F32, BF), (BF, None), (F32, None)])
@pytest.mark.parametrize("eight", [False, True])
def test_norm(d, T, dx, dr, eight):
    pad = -d % 8
    X = rows(T, d, dx, pad, seed=d)
    R = rows(T, d, dr, pad, seed=d + 1, scale=3.0) if dr else None
    w = 1 + 0.3 * torch.randn(d, device=DEV)
    r = api.sp_rms_norm(X, w, 1e-5, residual=R, out_dtype=F8 if eight else None, want_rstd=True)
    check_norm(X, R, w, 1e-5, r, eight)


@pytest.mark.parametrize("d, pad, shift", [(768, 1, 0), (768, 0, 1), (129, 0, 0), (4096, 3, 5)])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_layouts(d, pad, shift, eight, dtype):
    X, R = rows(9, d, dtype, pad, shift, 1), rows(9, d, dtype, pad + 2, shift + 1, 2)
    w = torch.randn(d + 1, device=DEV)[1:]
    out = torch.zeros(9, d + 5, device=DEV).to(F8 if eight else dtype)[:, :d]
    H = torch.zeros(9, d + 1, device=DEV, dtype=dtype)[:, 1:]
    r = api.sp_rms_norm(X, w, 1e-6, residual=R, h_out=H, out=out, want_rstd=True)
    assert r.H is H and r.Y is out
    check_norm(X, R, w, 1e-6, r, eight)


@pytest.mark.parametrize("d", [96, 1000, 4096, 40000])
def test_norm_in_place(d):
    X, R = rows(6, d, BF, -d % 8, seed=3), rows(6, d, F32, -d % 8, seed=4)
    want = api.sp_rms_norm(X, None, residual=R)
    x, r = X.clone(), R.clone()
    got = api.sp_rms_norm(x, None, residual=r, h_out=r, out=x)
    assert torch.equal(got.Y, want.Y) and torch.equal(got.H, want.H) and got.Y is x and got.H is r
    x = X.clone()
    got = api.sp_rms_norm(x, None, h_out=x)                      # h = x, written where it stands
    assert torch.equal(x, X) and torch.equal(got.Y, api.sp_rms_norm(X).Y)


@pytest.mark.parametrize("d", [100, 4096, 33000])
@pytest.mark.parametrize("eight", [False, True])
def test_norm_of_odd_values(d, eight):
    X = rows(7, d, F32, seed=5)
    X[0] = 0
    X[1, d // 2] = float("nan")
    X[2, d - 1] = float("inf")
    X[3] *= 1e-30                                                # (below eps: the row stays tiny)
    X[4] *= 1e15
    X[5] = 0
    X[5, 1] = 1e-22
    r = api.sp_rms_norm(X, None, 1e-5, out_dtype=F8 if eight else None, want_rstd=True)
    y = r.Y.float() * r.scale[:, None] if eight else r.Y
    assert (y[0] == 0).all() and y[1].isnan().all()
    assert y[2, d - 1].isnan() and (y[2, :d - 1] == 0).all()
    ok = [0, 3, 4, 5, 6]
    part = api.RmsNorm(r.Y[ok], None, r.scale[ok] if eight else None, r.rstd[ok])
    check_norm(X[ok], None, None, 1e-5, part, eight)


def test_norm_without_rows():
    r = api.sp_rms_norm(torch.empty(0, 64, device=DEV), want_rstd=True)
    assert r.Y.shape == (0, 64)
    dx, dw = api.sp_rms_norm_grad(torch.empty(0, 64, device=DEV), torch.empty(0, 64, device=DEV))
    assert dx.shape == (0, 64) and (dw == 0).all()


def grad64(dy, h, w, rstd, dh):
    dy, h, rstd = dy.double(), h.double(), rstd.double()[:, None]
    wdy = dy * (w.double() if w is not None else 1.0)
    dx = rstd * wdy - h * rstd ** 3 * (wdy * h).mean(1, keepdim=True)
    size = rstd * wdy.abs() + h.abs() * rstd ** 3 * (wdy * h).abs().mean(1, keepdim=True)
    if dh is not None:
        dx, size = dx + dh.double(), size + dh.double().abs()
    return dx, size, (dy * h * rstd).sum(0), (dy * h * rstd).abs().sum(0)


def check_grad(dY, H, w, rstd, dH, got, T, d):
    dx, size, dw, dw_size = grad64(dY, H, w, rstd, dH)
    assert got[0].dtype == H.dtype
    assert ((got[0].double() - dx).abs() <= dx.abs() * HALF[H.dtype] + size * additions(d) * 2.0 ** -24 + 1e-40).all()
    # (a block adds up at most its share of the rows one by one; products in fp32)
    assert ((got[1].double() - dw).abs() <= dw_size * (T / 148 + 32) * 2.0 ** -24 + 1e-40).all()


@pytest.mark.parametrize("d", [1, 8, 333, 512, 768, 1024, 2048, 2056, 4096, 6000, 8192, 12000, 16384, 20000])
@pytest.mark.parametrize("T", [1, 3, 70])
@pytest.mark.parametrize("dy, dh", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
def test_norm_grad(d, T, dy, dh):
    pad = -d % 8
    dY, H, dH = rows(T, d, dy, pad, seed=1), rows(T, d, dh, pad, seed=2, scale=2.0), rows(T, d, dh, pad, seed=3)
    w = 1 + 0.3 * torch.randn(d, device=DEV)
    rstd = (H.double().square().mean(1) + 1e-5).rsqrt().float()
    check_grad(dY, H, w, rstd, dH, api.sp_rms_norm_grad(dY, H, w, rstd, d_stream=dH), T, d)
    if T == 3:
        got = api.sp_rms_norm_grad(dY, H, None, None, 1e-5)         # no weight, rstd formed again, no gradient of the stream
        check_grad(dY, H, None, rstd, None, got, T, d)
        assert api.sp_rms_norm_grad(dY, H, None, None, 1e-5, want_weight=False)[1] is None


def test_norm_grad_of_many_rows_and_in_place():
    T, d = 5000, 776
    dY, H, dH = rows(T, d, BF, seed=1), rows(T, d, BF, seed=2), rows(T, d, BF, seed=3)
    w = torch.randn(d, device=DEV)
    rstd = (H.double().square().mean(1) + 1e-5).rsqrt().float()
    got = api.sp_rms_norm_grad(dY, H, w, rstd, d_stream=dH)
    check_grad(dY, H, w, rstd, dH, got, T, d)
    again = api.sp_rms_norm_grad(dY, H, w, rstd, d_stream=dH)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    a, b = dH.clone(), dY.clone()
    assert torch.equal(api.sp_rms_norm_grad(dY, H, w, rstd, d_stream=a, out=a)[0], got[0])
    assert torch.equal(api.sp_rms_norm_grad(b, H, w, rstd, d_stream=dH, out=b)[0], got[0])


@pytest.mark.parametrize("d, pad, shift", [(768, 1, 0), (768, 0, 1), (129, 0, 0)])
def test_norm_grad_layouts(d, pad, shift):
    T = 300
    dY, H, dH = rows(T, d, BF, pad, shift, 1), rows(T, d, F32, pad + 1, shift, 2), rows(T, d, F32, pad, shift + 1, 3)
    w = torch.randn(d + 1, device=DEV)[1:]
    rstd = (H.double().square().mean(1) + 1e-5).rsqrt().float()
    out = torch.zeros(T, d + 3, device=DEV)[:, 3:]
    check_grad(dY, H, w, rstd, dH, api.sp_rms_norm_grad(dY, H, w, rstd, d_stream=dH, out=out), T, d)


def test_norm_grad_against_differences():
    """The gradient of sum(c * y) + sum(e * h) against central differences of the forward call in fp32: with steps of 2^-6 the third derivative
    leaves about 2^-12, and the roundings of a sum of 3 x 40 products near 1 leave 2^-24 * 120 / 2^-5 = 2^-12."""
    T, d = 3, 40
    X, R = rows(T, d, F32, seed=6), rows(T, d, F32, seed=7)
    c, e = rows(T, d, F32, seed=8), rows(T, d, F32, seed=9)
    w = 1 + 0.3 * torch.randn(d, device=DEV)
    f = lambda x, u: float(((r := api.sp_rms_norm(x, u, 1e-5, residual=R)).Y.double() * c).sum() + (r.H.double() * e).sum())
    r = api.sp_rms_norm(X, w, 1e-5, residual=R, want_rstd=True)
    dx, dw = api.sp_rms_norm_grad(c, r.H, w, r.rstd, d_stream=e)
    step = 2.0 ** -6
    for t, j in ((0, 0), (1, 17), (2, 39)):
        p = torch.zeros_like(X)
        p[t, j] = step
        assert abs((f(X + p, w) - f(X - p, w)) / (2 * step) - float(dx[t, j])) < 2.0 ** -9
        q = torch.zeros_like(w)
        q[j] = step
        assert abs((f(X, w + q) - f(X, w - q)) / (2 * step) - float(dw[j])) < 2.0 ** -9
