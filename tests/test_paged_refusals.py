"""What sp_rms_norm, sp_rms_norm_grad, sp_linear_e4m3, sp_cache_append, sp_cache_read and sp_cache_attention refuse, on the host and before any
launch: the pointers below are never followed."""
import ctypes as C

import pytest
import torch

from paper_2510_03246_b200 import api, build

F32, BF16, F64, E4M3 = api.SP_F32, api.SP_BF16, api.SP_F64, api.SP_E4M3
OK, INVALID, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 9
P, Q = 0x1000, 0x9000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


def m(rows, cols, dtype=F32, ld=None, ptr=P):
    return api.SpMat(ptr, dtype, 0, rows, cols, cols if ld is None else ld)


def ref(x):
    return None if x is None else C.byref(x)


def norm(lib, X=m(4, 64), R=m(4, 64, ptr=0x2000), weight=P, eps=1e-5, H=m(4, 64, ptr=0x3000), Y=m(4, 64, ptr=0x4000), scale=None, rstd=None):
    return lib.sp_rms_norm(ref(X), ref(R), weight, eps, ref(H), ref(Y), scale, rstd, None)


def test_norm_refusals(lib):
    assert norm(lib, X=None) == INVALID and norm(lib, Y=None) == INVALID
    for eps in (-1.0, float("nan"), float("inf"), 1e31):
        assert norm(lib, eps=eps) == INVALID
    assert norm(lib, X=m(4, 64, F64)) == DTYPE and norm(lib, R=m(4, 64, F64)) == DTYPE and norm(lib, H=m(4, 64, BF16)) == DTYPE
    assert norm(lib, X=m(4, 64, E4M3)) == DTYPE and norm(lib, Y=m(4, 64, BF16)) == DTYPE
    assert norm(lib, Y=m(4, 64, E4M3)) == INVALID and norm(lib, scale=P) == INVALID          # scale goes with 8 bits
    for k in ("R", "H", "Y"):
        assert norm(lib, **{k: m(5, 64)}) == SHAPE and norm(lib, **{k: m(4, 63)}) == SHAPE
        assert norm(lib, **{k: m(4, 64, ld=63)}) == SHAPE and norm(lib, **{k: m(4, 64, ptr=None)}) == INVALID
    assert norm(lib, X=m(4, 64, ld=63)) == SHAPE and norm(lib, X=m(4, 0), R=None, H=None, Y=m(4, 0)) == SHAPE
    assert norm(lib, X=m(1 << 31, 64), R=None, H=None, Y=m(1 << 31, 64)) == SHAPE
    assert norm(lib, H=m(4, 64, ptr=0x4000)) == INVALID                                       # two outputs in one place
    assert norm(lib, H=m(4, 64, ld=65)) == INVALID                                            # X's place at another pitch
    assert norm(lib, R=m(4, 64, BF16, ptr=0x2000), H=m(4, 64, BF16)) == INVALID               # X's place, another type
    none = m(0, 64, ptr=None)
    assert norm(lib, X=none, R=None, H=None, Y=none) == OK


def grad(lib, dY=m(4, 64), H=m(4, 64, ptr=0x2000), weight=P, rstd=P, eps=1e-5, dH=m(4, 64, ptr=0x3000), dX=m(4, 64, ptr=0x4000), dw=P, ws=P,
         ws_bytes=1 << 20):
    return lib.sp_rms_norm_grad(ref(dY), ref(H), weight, rstd, eps, ref(dH), ref(dX), dw, ws, ws_bytes, None)


def test_norm_grad_refusals(lib):
    for k in ("dY", "H", "dX"):
        assert grad(lib, **{k: None}) == INVALID
    for k in ("H", "dH", "dX"):
        assert grad(lib, **{k: m(5, 64)}) == SHAPE and grad(lib, **{k: m(4, 64, ld=63)}) == SHAPE
        assert grad(lib, **{k: m(4, 64, BF16)}) == DTYPE and grad(lib, **{k: m(4, 64, ptr=None)}) == INVALID
    assert grad(lib, dY=m(4, 64, E4M3)) == DTYPE and grad(lib, eps=-1.0) == INVALID
    need = lib.sp_rms_norm_grad_bytes(4, 64)
    assert need >= 64 * 4
    assert grad(lib, ws=None) == WORKSPACE and grad(lib, ws_bytes=need - 1) == WORKSPACE and grad(lib, ws=0x1010) == ALIGN
    assert grad(lib, dX=m(4, 64, ld=70)) == INVALID                                           # dY's place at another pitch
    assert lib.sp_rms_norm_grad_bytes(0, 64) == 0 and lib.sp_rms_norm_grad_bytes(4, 0) == 0
    none = m(0, 64, ptr=None)
    assert grad(lib, dY=none, H=none, dH=None, dX=none, dw=None) == OK


def linear(lib, X=m(4, 64, E4M3), xs=P, W=m(8, 64, E4M3), ws=P, bias=None, act=0, other=None, combine=0, Y=m(4, 8, BF16)):
    return lib.sp_linear_e4m3(ref(X), xs, ref(W), ws, bias, act, ref(other), combine, ref(Y), None, None)


def test_linear_refusals(lib):
    for k in ("X", "W", "Y"):
        assert linear(lib, **{k: None}) == INVALID
    assert linear(lib, xs=None) == INVALID and linear(lib, ws=None) == INVALID
    assert linear(lib, act=4) == INVALID and linear(lib, act=-1) == INVALID and linear(lib, combine=2) == INVALID
    assert linear(lib, X=m(4, 64, BF16)) == DTYPE and linear(lib, W=m(8, 64, F32)) == DTYPE and linear(lib, Y=m(4, 8, E4M3)) == DTYPE
    assert linear(lib, other=m(4, 8, F32)) == DTYPE
    assert linear(lib, W=m(8, 63, E4M3)) == SHAPE and linear(lib, Y=m(4, 9, BF16)) == SHAPE and linear(lib, other=m(5, 8, BF16)) == SHAPE
    assert linear(lib, X=m(4, 64, E4M3, ld=63)) == SHAPE and linear(lib, X=m(4, 0, E4M3), W=m(8, 0, E4M3)) == SHAPE
    assert linear(lib, X=m(4, 64, E4M3, ld=72)) == ALIGN and linear(lib, W=m(8, 64, E4M3, ld=65)) == ALIGN
    assert linear(lib, X=m(4, 64, E4M3, ptr=0x1008)) == ALIGN and linear(lib, W=m(8, 64, E4M3, ptr=0x1001)) == ALIGN
    assert linear(lib, other=m(4, 8, BF16), Y=m(4, 8, BF16, ld=9)) == INVALID
    assert linear(lib, X=m(4, 64, E4M3, ptr=None)) == INVALID
    assert linear(lib, X=m(0, 64, E4M3, ptr=None), Y=m(0, 8, BF16, ptr=None), xs=None) == OK
    # types of the other calls stay what they were
    assert lib.sp_linear(ref(m(4, 64, E4M3)), ref(m(8, 64, E4M3)), None, 0, None, 0, ref(m(4, 8)), None, None) == DTYPE
    x = m(8, 8, E4M3)
    assert lib.sp_gemm(0, 0, 8, 8, 8, 1.0, ref(x), ref(x), 0.0, ref(m(8, 8)), 0, 0, None, None) == DTYPE


def kv(four=False, **kw):
    d_head = kw.get("d_head", 64)
    n_kv, page_len = kw.get("n_kv_heads", 2), kw.get("page_len", 16)
    tokens = n_kv * page_len
    f = dict(k=P, v=P, k_scale=P if four else None, v_scale=P if four else None, step=tokens * (d_head // 2 if four else 2 * d_head),
             scale_step=tokens * (d_head // 64) * 4 if four else 0, table=P, lens=P, table_ld=5, max_pages=5, n_seq=3,
             kind=api.SP_CACHE_4BIT if four else api.SP_CACHE_BF16, n_pages=9, page_len=16, n_kv_heads=2, d_head=64)
    f.update(kw)
    return api.SpKvCache(**f)


def append(lib, c, **kw):
    f = dict(Q=m(6, 256), K=m(6, 128), V=m(6, 128), Q_out=m(6, 256, ptr=0x2000), K_out=m(6, 128, ptr=0x3000), cu=P, positions=None, inv_freq=P,
             n_heads=4, turned=64, neighbours=0)
    f.update(kw)
    return lib.sp_cache_append(ref(c), C.byref(api.SpCacheAppendArgs(**f)), None, None)


def read(lib, c, cu=P, K=m(6, 128), V=m(6, 128, ptr=0x2000)):
    return lib.sp_cache_read(ref(c), cu, ref(K), ref(V), None, None)


def attend(lib, c, Qm=m(6, 256), cu=P, n_heads=4, scale=0.125, max_keys=0, O=m(6, 256, ptr=0x2000), ws=0x4000, ws_bytes=1 << 40):
    return lib.sp_cache_attention(ref(c), ref(Qm), cu, n_heads, 1, scale, max_keys, ref(O), None, None, ws, ws_bytes, None)


@pytest.mark.parametrize("four", [False, True])
def test_caches_that_are_refused(lib, four):
    calls = (append, read, attend)
    for bad, code in ((dict(kind=2), INVALID), (dict(kind=-1), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID),
                      (dict(lens=None), INVALID), (dict(n_kv_heads=0), SHAPE), (dict(n_seq=-1), SHAPE), (dict(n_pages=0), SHAPE),
                      (dict(page_len=8), SHAPE), (dict(page_len=24), SHAPE), (dict(page_len=0), SHAPE), (dict(max_pages=-1), SHAPE),
                      (dict(table_ld=4), SHAPE), (dict(max_pages=1 << 28, table_ld=1 << 28), SHAPE), (dict(d_head=0), SHAPE),
                      (dict(d_head=192), UNSUPPORTED), (dict(d_head=72), UNSUPPORTED), (dict(step=2048 + 64), SHAPE), (dict(step=128), SHAPE),
                      (dict(step=1 << 39), SHAPE), (dict(k=0x1008), ALIGN), (dict(v=0x1008), ALIGN)):
        for call in calls:
            assert call(lib, kv(four, **bad)) == code, (bad, call.__name__)
    if four:
        for bad, code in ((dict(k_scale=None), INVALID), (dict(scale_step=32), SHAPE), (dict(scale_step=160), SHAPE), (dict(v_scale=0x1008), ALIGN),
                          (dict(d_head=80), UNSUPPORTED), (dict(d_head=96), UNSUPPORTED)):
            for call in calls:
                assert call(lib, kv(four, **bad)) == code, (bad, call.__name__)
    for call in calls:
        assert call(lib, None) == INVALID
        if call is not append:
            assert call(lib, kv(four, k=None)) == INVALID


def test_append_refusals(lib):
    c = kv()
    assert lib.sp_cache_append(ref(c), None, None, None) == INVALID
    for k, cols in (("K", 128), ("V", 128), ("Q", 256), ("Q_out", 256), ("K_out", 128)):
        assert append(lib, c, **{k: m(6, cols, BF16, ptr=0x7000)}) == DTYPE, k
        assert append(lib, c, **{k: m(7, cols, ptr=0x7000)}) == SHAPE and append(lib, c, **{k: m(6, cols + 64, ptr=0x7000)}) == SHAPE, k
        assert append(lib, c, **{k: m(6, cols, ld=cols - 1, ptr=0x7000)}) == SHAPE, k
    assert append(lib, c, K=m(6, 128, F64)) == DTYPE
    for k in ("K", "V", "Q", "Q_out"):
        assert append(lib, c, **{k: m(6, 256 if k[0] == "Q" else 128, ptr=None)}) == INVALID, k
    assert append(lib, c, cu=None) == INVALID and append(lib, c, inv_freq=None) == INVALID
    for turned in (-16, 8, 80, 65):
        assert append(lib, c, turned=turned) == SHAPE
    assert append(lib, c, K_out=m(6, 128)) == INVALID                          # in K's place
    assert append(lib, c, Q_out=m(6, 256, ld=260)) == INVALID                  # in Q's place at another pitch
    assert append(lib, c, n_heads=0) == SHAPE and append(lib, c, n_heads=3) == SHAPE
    none = m(0, 128, ptr=None)
    assert append(lib, c, K=none, V=none, Q=m(0, 0, ptr=None), Q_out=m(0, 0, ptr=None), K_out=m(0, 0, ptr=None), cu=None) == OK
    assert append(lib, kv(n_seq=0, table=None, lens=None)) == OK


def test_read_refusals(lib):
    c = kv()
    assert read(lib, c, cu=None) == INVALID and read(lib, c, K=None) == INVALID and read(lib, c, V=m(6, 128)) == INVALID
    assert read(lib, c, K=m(6, 128, F64)) == DTYPE and read(lib, c, V=m(6, 128, BF16, ptr=0x2000)) == DTYPE
    assert read(lib, c, K=m(6, 64)) == SHAPE and read(lib, c, V=m(5, 128, ptr=0x2000)) == SHAPE and read(lib, c, K=m(6, 128, ld=100)) == SHAPE
    assert read(lib, c, K=m(0, 128, ptr=None), V=m(0, 128, ptr=None), cu=None) == OK


@pytest.mark.parametrize("rows", [6, 600])
def test_attention_refusals(lib, rows):
    c = kv()
    q, o = m(rows, 256), m(rows, 256, ptr=0x2000)
    assert attend(lib, c, None) == INVALID and attend(lib, c, q, O=None) == INVALID and attend(lib, c, q, cu=None, O=o) == INVALID
    assert attend(lib, c, m(rows, 256, F64), O=o) == DTYPE and attend(lib, c, q, O=m(rows, 256, BF16)) == DTYPE
    assert attend(lib, c, q, O=m(rows + 1, 256)) == SHAPE and attend(lib, c, m(rows, 192), O=o) == SHAPE
    assert attend(lib, c, m(rows, 256, ld=250), O=o) == SHAPE and attend(lib, c, q, n_heads=3, O=o) == SHAPE and attend(lib, c, q, n_heads=0, O=o) == SHAPE
    assert attend(lib, c, q, max_keys=-1, O=o) == SHAPE
    for scale in (0.0, -1.0, float("nan"), 1e31, 1e-31):
        assert attend(lib, c, q, scale=scale, O=o) == INVALID
    need = lib.sp_cache_attention_bytes(rows, 3, 4, 2, 64, F32, 5, 16, 0)
    assert need > 0
    assert attend(lib, c, q, O=o, ws=None) == WORKSPACE and attend(lib, c, q, O=o, ws_bytes=need - 1) == WORKSPACE
    assert attend(lib, c, q, O=o, ws=0x4010) == ALIGN
    assert attend(lib, c, m(0, 256, ptr=None), O=m(0, 256, ptr=None), cu=None, ws=None) == OK
    assert attend(lib, kv(n_seq=0, table=None, lens=None), q, O=o, cu=None, ws=None) == OK


def test_attention_workspace_sizes(lib):
    bytes_of = lib.sp_cache_attention_bytes
    few = bytes_of(16, 16, 32, 8, 128, BF16, 512, 64, 0)
    assert 0 < few <= 16 << 20 and few == bytes_of(16, 16, 32, 8, 128, BF16, 1 << 20, 64, 0)      # not a matter of the table's size
    many = bytes_of(512, 1, 32, 8, 128, BF16, 512, 64, 16384)
    assert many >= 2 * 16384 * 1024 * 2 and bytes_of(512, 1, 32, 8, 128, BF16, 512, 64, 0) > many
    for bad in ((0, 16, 32, 8, 128, BF16, 512, 64, 0), (16, 0, 32, 8, 128, BF16, 512, 64, 0), (16, 16, 30, 8, 128, BF16, 512, 64, 0),
                (16, 16, 32, 8, 129, BF16, 512, 64, 0), (16, 16, 32, 8, 128, BF16, 1 << 25, 64, 0)):
        assert bytes_of(*bad) == 0
    # more keys than can be opened
    assert bytes_of(100000, 1000, 32, 8, 128, BF16, 1 << 20, 64, 0) == 0


def test_the_binding_refuses_tensors_off_the_device():
    """Through Python: CPU tensors, and arguments that are none."""
    x = torch.zeros(4, 64)
    i = torch.zeros(3, dtype=torch.int32)
    pages = api.KvPages.empty(4, 1, 16, 64, device="cpu")
    with pytest.raises(RuntimeError):
        api.sp_rms_norm(x)
    with pytest.raises(RuntimeError):
        api.sp_rms_norm_grad(x, x)
    with pytest.raises(RuntimeError):
        api.sp_linear_e4m3(x.to(torch.float8_e4m3fn), None, x.to(torch.float8_e4m3fn), None)
    with pytest.raises(RuntimeError):
        api.sp_cache_append(pages, x, x, i, i.view(1, 3), i)
    with pytest.raises(RuntimeError):
        api.sp_cache_read(pages, i, i.view(1, 3), i, 4)
    with pytest.raises(RuntimeError):
        api.sp_cache_attention(x, pages, i, i.view(1, 3), i, 1)
    with pytest.raises(TypeError):
        api.sp_rms_norm("x", out_dtype=None)
    for bad in (torch.bfloat16, torch.float16):
        with pytest.raises(ValueError):
            api.sp_rms_norm(x, out_dtype=bad)
    with pytest.raises(ValueError):
        api.sp_linear_e4m3(x, None, x, None, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        api.sp_cache_read(pages, i, i.view(1, 3), i, 4, dtype=torch.float16)
