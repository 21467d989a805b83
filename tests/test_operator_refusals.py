"""What sp_attention, sp_linear, sp_token_logprobs and sp_token_logprobs_grad refuse, on the host and before any launch: the pointers below are never
followed."""
import ctypes as C

import pytest

from paper_2510_03246_b200 import api, build

F32, BF16, F64 = api.SP_F32, api.SP_BF16, api.SP_F64
OK, INVALID, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 9
P = 0x1000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


def m(rows, cols, dtype=F32, ld=None, ptr=P):
    return api.SpMat(ptr, dtype, 0, rows, cols, cols if ld is None else ld)


def attention(lib, ws=None, ws_bytes=0, **kw):
    f = dict(Q=m(1024, 256), K=m(1024, 128), V=m(1024, 128), O=m(1024, 256), cu_q=P, cu_k=P, lse=None, n_seq=600, n_heads=4,
             n_kv_heads=2, causal=1, scale=0.125)
    f.update(kw)
    return lib.sp_attention(C.byref(api.SpAttentionArgs(**f)), None, ws, ws_bytes, None)


def test_attention_refusals(lib):
    assert lib.sp_attention(None, None, None, 0, None) == INVALID
    for name in "QKVO":
        shape = (1024, 256) if name in "QO" else (1024, 128)
        assert attention(lib, **{name: m(*shape, dtype=BF16)}) == DTYPE
        assert attention(lib, **{name: m(*shape, ld=shape[1] - 1)}) == SHAPE
        assert attention(lib, **{name: m(*shape, ptr=None)}) == INVALID
        assert attention(lib, **{name: m(shape[0], shape[1] + 4)}) == SHAPE
    assert attention(lib, Q=m(1024, 256, F64)) == DTYPE
    assert attention(lib, O=m(1000, 256)) == SHAPE and attention(lib, V=m(1000, 128)) == SHAPE
    assert attention(lib, n_kv_heads=3) == SHAPE and attention(lib, n_heads=0) == SHAPE
    assert attention(lib, n_kv_heads=0) == SHAPE and attention(lib, n_seq=-1) == SHAPE
    assert attention(lib, n_heads=3, n_kv_heads=3) == SHAPE                    # 256 columns are not 3 heads
    assert attention(lib, Q=m((1 << 30) + 1, 256), O=m((1 << 30) + 1, 256)) == SHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e31, 1e-31):
        assert attention(lib, scale=scale) == INVALID
    assert attention(lib, cu_q=None) == INVALID and attention(lib, cu_k=None) == INVALID
    wide = dict(Q=m(8, 129), O=m(8, 129), K=m(8, 129), V=m(8, 129), n_heads=1, n_kv_heads=1)
    assert attention(lib, **wide) == UNSUPPORTED
    # a call whose keys are cut needs its workspace, aligned
    long = dict(Q=m(1, 256), O=m(1, 256), K=m(9000, 128), V=m(9000, 128), n_seq=1)
    need = lib.sp_attention_workspace_bytes(1, 9000, 1, 4, 2, 64, F32)
    assert need > 0
    assert attention(lib, **long) == WORKSPACE
    assert attention(lib, ws=C.c_void_p(0x1000), ws_bytes=need - 1, **long) == WORKSPACE
    assert attention(lib, ws=C.c_void_p(0x1010), ws_bytes=need, **long) == ALIGN
    # nothing to do: no pointer is needed
    none = m(0, 256, ptr=None)
    assert attention(lib, Q=none, O=none, cu_q=None) == OK
    assert attention(lib, n_seq=0, cu_q=None, cu_k=None) == OK


def test_attention_workspace(lib):
    w = lambda *a: lib.sp_attention_workspace_bytes(*a, BF16)
    assert w(128 * 2048, 128 * 2048, 128, 32, 32, 128) == 0                    # rows enough to fill the GPU
    assert w(16, 16 * 32768, 16, 32, 8, 128) > 0
    assert w(0, 100, 1, 8, 8, 64) == 0 and w(1, 0, 1, 8, 8, 64) == 0 and w(1, 200, 1, 8, 8, 64) == 0
    assert w(1, 1 << 24, 0, 8, 8, 64) == 0 and w(1, 1 << 24, 1, 8, 3, 64) == 0 and w(-1, 100, 1, 8, 8, 64) == 0
    assert w(64, 1 << 30, 64, 32, 8, 128) < 2 << 30


def linear(lib, X=None, W=None, other=None, Y=None, bias=None, act=0, combine=0):
    X, W, Y = X or m(10, 64), W or m(32, 64), Y or m(10, 32)
    return lib.sp_linear(C.byref(X), C.byref(W), bias, act, C.byref(other) if other else None, combine, C.byref(Y), None, None)


def test_linear_refusals(lib):
    assert lib.sp_linear(None, None, None, 0, None, 0, None, None, None) == INVALID
    assert linear(lib, act=4) == INVALID and linear(lib, act=-1) == INVALID
    assert linear(lib, combine=2) == INVALID and linear(lib, combine=-1) == INVALID
    assert linear(lib, X=m(10, 64, F64)) == DTYPE and linear(lib, W=m(32, 64, BF16)) == DTYPE
    assert linear(lib, Y=m(10, 32, BF16)) == DTYPE and linear(lib, other=m(10, 32, BF16)) == DTYPE
    assert linear(lib, W=m(32, 63)) == SHAPE and linear(lib, Y=m(9, 32)) == SHAPE and linear(lib, Y=m(10, 31)) == SHAPE
    assert linear(lib, other=m(10, 31)) == SHAPE and linear(lib, other=m(9, 32)) == SHAPE
    assert linear(lib, X=m(10, 64, ld=63)) == SHAPE and linear(lib, W=m(32, 64, ld=10)) == SHAPE
    assert linear(lib, Y=m(10, 32, ld=31)) == SHAPE and linear(lib, other=m(10, 32, ld=31)) == SHAPE
    assert linear(lib, X=m(10, 0), W=m(32, 0)) == SHAPE
    assert linear(lib, X=m((1 << 22) + 1, 64), Y=m((1 << 22) + 1, 32)) == SHAPE
    assert linear(lib, X=m(10, 64, ptr=None)) == INVALID and linear(lib, W=m(32, 64, ptr=None)) == INVALID
    assert linear(lib, Y=m(10, 32, ptr=None)) == INVALID and linear(lib, other=m(10, 32, ptr=None)) == INVALID
    assert linear(lib, other=m(10, 32, ld=40), Y=m(10, 32, ld=48)) == INVALID  # the same values at another pitch
    assert linear(lib, X=m(0, 64, ptr=None), Y=m(0, 32, ptr=None)) == OK


def logprobs(lib, x, targets=P, scale=1.0, n_alts=0, logp=P, lse=P, entropy=None, ids=None, alts=None):
    return lib.sp_token_logprobs(C.byref(x), targets, scale, n_alts, logp, lse, entropy, ids, alts, None, None)


def test_logprob_refusals(lib):
    assert lib.sp_token_logprobs(None, P, 1.0, 0, P, P, None, None, None, None, None) == INVALID
    assert logprobs(lib, m(4, 100, F64)) == DTYPE
    assert logprobs(lib, m(4, 100, ld=99)) == SHAPE and logprobs(lib, m(-1, 100)) == SHAPE
    assert logprobs(lib, m(4, 0)) == SHAPE and logprobs(lib, m(4, (1 << 30) + 1)) == SHAPE
    assert logprobs(lib, m(1 << 29, 10)) == SHAPE
    for n in (-1, 33):
        assert logprobs(lib, m(4, 100), n_alts=n, ids=P) == SHAPE
    assert logprobs(lib, m(4, 3), n_alts=4, ids=P) == SHAPE                    # more alternatives than logits
    assert logprobs(lib, m(4, 100), n_alts=2) == INVALID and logprobs(lib, m(4, 100), ids=P) == INVALID
    for scale in (0.0, -2.0, float("nan"), float("inf"), 1e31, 1e-31):
        assert logprobs(lib, m(4, 100), scale=scale) == INVALID
    assert logprobs(lib, m(4, 100), targets=None) == INVALID
    assert logprobs(lib, m(4, 100), logp=None, lse=None) == INVALID
    assert logprobs(lib, m(4, 100, ptr=None)) == INVALID
    assert logprobs(lib, m(0, 100, ptr=None)) == OK


def grad(lib, x, d, targets=P, scale=1.0, lse=P, entropy=P, gl=P, gh=None):
    return lib.sp_token_logprobs_grad(C.byref(x), targets, scale, lse, entropy, gl, gh, C.byref(d), None)


def test_gradient_refusals(lib):
    x = m(4, 100)
    assert lib.sp_token_logprobs_grad(None, P, 1.0, P, P, P, P, None, None) == INVALID
    assert grad(lib, m(4, 100, F64), m(4, 100, F64)) == DTYPE and grad(lib, x, m(4, 100, BF16)) == DTYPE
    assert grad(lib, x, m(4, 99)) == SHAPE and grad(lib, x, m(3, 100)) == SHAPE and grad(lib, x, m(4, 100, ld=10)) == SHAPE
    assert grad(lib, x, x, gl=None) == INVALID and grad(lib, x, x, targets=None) == INVALID
    assert grad(lib, x, x, lse=None) == INVALID and grad(lib, x, x, gh=P, entropy=None) == INVALID
    assert grad(lib, x, m(4, 100, ptr=None)) == INVALID
    assert grad(lib, x, m(4, 100, ld=104)) == INVALID                          # in place at another pitch
    for scale in (0.0, -2.0, float("nan"), float("inf"), 1e31, 1e-31):
        assert grad(lib, x, x, scale=scale) == INVALID
    assert grad(lib, m(0, 100, ptr=None), m(0, 100, ptr=None)) == OK


def test_binding_refuses_cpu_tensors_in_attention(lib):
    import torch
    x, cu = torch.zeros(4, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        api.sp_attention(x, x, x, cu, cu, 1)


def test_binding_refuses_cpu_tensors_in_linear(lib):
    import torch
    with pytest.raises(RuntimeError):
        api.sp_linear(torch.zeros(4, 8), torch.zeros(4, 8))


def test_binding_refuses_cpu_tensors_in_logprobs(lib):
    import torch
    x = torch.zeros(4, 8)
    for call in (lambda: api.sp_token_logprobs(x), lambda: api.sp_token_logprobs_grad(x, None, x[:, 0], x[:, 0])):
        with pytest.raises(RuntimeError):
            call()
