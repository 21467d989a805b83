"""Widths that are no multiple of eight: what sp_rms_norm and sp_rms_norm_grad allocate has rows that start on 16 bytes, so that calls with such
inputs keep each row in registers, and the rows' ends are right there, several rows of a block side by side and one after another."""
import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def rows(T, d, dtype, seed):
    t = api.rows_of_16_bytes(T, d, dtype, DEV)
    t.copy_(torch.randn(T, d, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
    return t


def aligned(t):
    return t.data_ptr() % 16 == 0 and (t.shape[0] < 2 or t.stride(0) * t.element_size() % 16 == 0)


@pytest.mark.parametrize("d", [1, 5, 97, 333, 1027, 2049, 4093, 8189])
@pytest.mark.parametrize("T", [2, 3, 70, 700])
@pytest.mark.parametrize("dy, dh", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
def test_rows_that_end_inside_a_chunk(d, T, dy, dh):
    X, R, w = rows(T, d, dy, 1), rows(T, d, dh, 2), 1 + 0.2 * torch.randn(d, device=DEV)
    r = api.sp_rms_norm(X, w, residual=R, want_rstd=True)
    assert aligned(r.H) and aligned(r.Y) and r.H.shape == (T, d)
    h = X.double() + R.double()
    assert ((r.H.double() - h).abs() <= h.abs() * HALF[dh] + 2.0 ** -24 * (X.double().abs() + R.double().abs())).all()
    G, S = rows(T, d, dy, 3), rows(T, d, dh, 4)
    dX, dw = api.sp_rms_norm_grad(G, r.H, w, r.rstd, d_stream=S)
    assert aligned(dX) and dX.shape == (T, d) and dX.dtype == dh
    H, rstd, u = r.H.double(), r.rstd.double()[:, None], G.double() * w.double()
    mean = (u * H).mean(1, keepdim=True)
    want = rstd * (u - H * rstd.square() * mean) + S.double()
    # some 64 additions of fp32 on the way of a value to a row's sum, four roundings after it, the result's own
    near = rstd * (u.abs() * 4 + H.abs() * rstd.square() * (u * H).abs().mean(1, keepdim=True) * 68) * 2.0 ** -24 + 2.0 ** -24 * S.double().abs()
    assert ((dX.double() - want).abs() <= want.abs() * HALF[dh] + near).all()
    terms = G.double() * H * rstd
    # a block adds up its rows (at most all T) in fp32
    assert ((dw.double() - terms.sum(0)).abs() <= terms.abs().sum(0) * (T + 4) * 2.0 ** -24 + 1e-30).all()
    none, again = api.sp_rms_norm_grad(G, r.H, w, r.rstd, d_stream=S)
    assert torch.equal(dX, none) and torch.equal(dw, again)


@pytest.mark.parametrize("T, d", [(1, 64), (7, 97), (295, 333), (296, 333), (297, 64), (3000, 97), (149, 9000)])
def test_gradient_of_rows_on_any_address(T, d):
    """One row of a block at a time, more rows than blocks: the weight's gradient of all of them."""
    G, H = (torch.randn(T, d + 1, generator=torch.Generator(device=DEV).manual_seed(s), device=DEV)[:, 1:] for s in (5, 6))
    w = 1 + 0.2 * torch.randn(d, device=DEV)
    need = api.lib().sp_rms_norm_grad_bytes(T, d)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    dX, dw = api.sp_rms_norm_grad(G, H, w, ws=ws[:need])
    assert (ws[need:] == 255).all()
    h, g = H.double(), G.double()
    rstd = (h.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    u = g * w.double()
    want = rstd * (u - h * rstd.square() * (u * h).mean(1, keepdim=True))
    near = rstd * (u.abs() * (4 + d / 512 + 64) + h.abs() * rstd.square() * (u * h).abs().mean(1, keepdim=True) * (68 + d / 512)) * 2.0 ** -24
    assert ((dX.double() - want).abs() <= want.abs() * 2.0 ** -24 + 3 * near).all()
    terms = (g * h * rstd).abs().sum(0)
    assert ((dw.double() - (g * h * rstd).sum(0)).abs() <= terms * (T + 4 + d / 512 + 64) * 2.0 ** -24 + 1e-30).all()
