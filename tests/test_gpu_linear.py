"""sp_linear against the definition in 64 bits.

Tolerances: a sum of K products in fp32 is off by at most K 2^-23 sum |x w| (one step per addition, chopped or rounded), the
bias adds one; fp32 mode sums in fp64 (K 2^-52).  The activations' slopes are at most 1.13 and their own error is within
2^-16 of their value for |v| < 100 (exponential of an argument rounded in fp32, erfc); then one operation with `other` and one
rounding to the storage type (half a step)."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ACTS = {api.SP_LINEAR_NONE: lambda v: v, api.SP_LINEAR_RELU: torch.relu, api.SP_LINEAR_SILU: torch.nn.functional.silu,
        api.SP_LINEAR_GELU: torch.nn.functional.gelu}


def inputs(T, K, N, dtype, seed=0, wide=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    make = (lambda r, c: api.rows_of_16_bytes(r, c, dtype, DEV)) if wide else \
           (lambda r, c: torch.empty(r, c, dtype=dtype, device=DEV))
    x, w, o = make(T, K), make(N, K), make(T, N)
    x.copy_(torch.randn(T, K, generator=g, device=DEV))
    w.copy_(torch.randn(N, K, generator=g, device=DEV) / math.sqrt(K))
    o.copy_(torch.randn(T, N, generator=g, device=DEV))
    return x, w, o, torch.randn(N, generator=g, device=DEV)


def check(x, w, bias=None, act=0, other=None, combine=0, out=None, out_dtype=None):
    K = x.shape[1]
    before = other.clone() if other is not None else None
    y = api.sp_linear(x, w, bias=bias, act=act, other=other, combine=combine, out=out, out_dtype=out_dtype)
    v = x.double() @ w.double().T
    e = (x.double().abs() @ w.double().abs().T) * K * 2.0 ** (-23 if x.dtype == torch.bfloat16 else -52)
    if bias is not None:
        v = v + bias.double()
        e = e + v.abs() * 2.0 ** -23
    v = ACTS[act](v)
    e = 1.13 * e + (v.abs() * 2.0 ** -16 if act > 1 else 0.0)
    if before is not None:
        if combine == api.SP_COMBINE_MUL:
            v, e = v * before.double(), e * before.double().abs()
        else:
            v = v + before.double()
    tol = e * 1.01 + (HALF[y.dtype] + 2.0 ** -22) * v.abs() + 1e-30
    err = (y.double() - v).abs()
    assert torch.isfinite(y).all() and (err <= tol).all(), float((err / tol).max())
    return y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (1, 768, 1536), (2, 65, 129), (5, 4096, 257), (16, 1000, 4097), (17, 64, 64),
                                   (33, 333, 1311), (128, 128, 128), (300, 1311, 520), (1000, 777, 1024), (257, 2048, 3303)])
def test_sizes(dtype, T, K, N):
    x, w, o, b = inputs(T, K, N, dtype, seed=T + N)
    check(x, w)
    check(x, w, bias=b, act=api.SP_LINEAR_RELU)
    check(x, w, bias=b, other=o)
    check(x, w, act=api.SP_LINEAR_SILU, other=o, combine=api.SP_COMBINE_MUL)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("N", [256, 250])
def test_epilogues(dtype, act, T, N):
    x, w, o, b = inputs(T, 192, N, dtype)
    x[0] *= 60                                                     # far into both tails of the activation
    for bias in (None, b):
        for other, combine in ((None, 0), (o, api.SP_COMBINE_ADD), (o, api.SP_COMBINE_MUL)):
            check(x, w, bias=bias, act=act, other=other, combine=combine)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("T", [4, 160])
def test_fp32_result_of_bf16_operands(act, T):
    for N in (256, 255):
        x, w, _, b = inputs(T, 320, N, torch.bfloat16)
        o = torch.randn(T, N, device=DEV)
        y = check(x, w, bias=b, act=act, out_dtype=torch.float32)
        assert y.dtype == torch.float32
        check(x, w, bias=b, act=act, other=o, out_dtype=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [6, 190])
@pytest.mark.parametrize("combine", [api.SP_COMBINE_ADD, api.SP_COMBINE_MUL])
def test_other_in_place(dtype, T, combine):
    x, w, o, b = inputs(T, 96, 264, dtype)
    y = check(x, w, bias=b, other=o, combine=combine, out=o)
    assert y.data_ptr() == o.data_ptr()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [5, 140])
def test_pitches_and_what_lies_beside_the_result(dtype, T):
    x, w, o, b = inputs(T, 77, 131, dtype, wide=False)             # contiguous odd widths
    check(x, w, bias=b, other=o)
    for start, N in ((0, 131), (8, 131), (3, 128), (8, 136)):
        x, w, o, b = inputs(T, 77, N, dtype)
        buf = torch.full((T, 160), 7.0, dtype=dtype, device=DEV)
        check(x, w, bias=b, other=o, out=buf[:, start:start + N])
        assert (buf[:, :start] == 7).all() and (buf[:, start + N:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [4, 150])
def test_values_beside_a_ragged_width_do_not_enter(dtype, T):
    """What stands in the rows of X and W beyond the width (there to align them) is no part of the product."""
    bx = torch.full((T, 80), math.nan, dtype=dtype, device=DEV)
    bw = torch.full((50, 80), math.nan, dtype=dtype, device=DEV)
    x, w, _, _ = inputs(T, 77, 50, dtype)
    bx[:, :77], bw[:, :77] = x, w
    check(bx[:, :77], bw[:, :77])


@pytest.mark.parametrize("T", [3, 130])
def test_infinities_and_nan(T):
    x, w, _, b = inputs(T, 64, 128, torch.bfloat16)
    w.zero_()
    w[:, 0] = 1
    x[:, 0] = 1
    b[0], b[1], b[2] = math.nan, math.inf, -math.inf
    y = {a: api.sp_linear(x, w, bias=b, act=a) for a in ACTS}
    for a in ACTS:
        assert torch.isnan(y[a][:, 0]).all() and (y[a][:, 1] == math.inf).all() and torch.isfinite(y[a][:, 3:]).all()
    assert (y[0][:, 2] == -math.inf).all()
    for a in (1, 2, 3):
        assert (y[a][:, 2] == 0).all()


def test_nothing_to_do():
    for T, N in ((0, 5), (5, 0)):
        y = api.sp_linear(torch.zeros(T, 8, device=DEV), torch.zeros(N, 8, device=DEV))
        assert y.shape == (T, N)


@pytest.mark.parametrize("T", [2, 300])
def test_another_stream_and_a_captured_call(T):
    x, w, o, b = inputs(T, 512, 640, torch.bfloat16)
    want = check(x, w, bias=b, act=1, other=o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = api.sp_linear(x, w, bias=b, act=1, other=o)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = api.sp_linear(x, w, bias=b, act=1, other=o)
    z.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, want)


@pytest.mark.parametrize("T,K,N", [(17, 768, 1536), (24, 1311, 520), (32, 2048, 8192), (32, 320, 8200), (25, 9, 3)])
def test_up_to_32_rows(T, K, N):
    x, w, o, b = inputs(T, K, N, torch.bfloat16, seed=T)
    check(x, w)
    check(x, w, bias=b, act=api.SP_LINEAR_SILU, other=o, combine=api.SP_COMBINE_MUL)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,N", [(1, 1), (1, 70), (50, 1)])
def test_a_single_row_has_no_pitch(dtype, T, N):
    K = 77
    x, w, _, _ = inputs(T, K, N, dtype)
    want = check(x, w)
    y = torch.zeros(T, N, dtype=dtype, device=DEV)
    code = api._DTYPES[dtype]
    m = lambda t, r, c: api.SpMat(t.data_ptr(), code, 0, r, c, t.stride(0) if r > 1 else 3)
    X, W, Y = m(x, T, K), m(w, N, K), m(y, T, N)
    assert api.lib().sp_linear(api.C.byref(X), api.C.byref(W), None, 0, None, 0, api.C.byref(Y), None,
                               torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y, want)


@pytest.mark.parametrize("T,K,N", [(1, 5, 1), (8, 16, 17), (9, 512, 33), (16, 2047, 100), (33, 700, 65), (64, 4096, 48), (129, 512, 96),
                                   (512, 530, 40), (513, 530, 40), (200, 511, 70)])
def test_few_rows_in_fp32(T, K, N):
    """Every group of rows, whole and ragged pieces of K, on both sides of the choice of form."""
    for wide in (True, False):
        x, w, o, b = inputs(T, K, N, torch.float32, seed=T, wide=wide)
        check(x, w)
        check(x, w, bias=b, act=api.SP_LINEAR_GELU, other=o, combine=api.SP_COMBINE_MUL)


@pytest.mark.parametrize("T", [1, 40])
def test_infinities_and_subnormal_values_in_fp32(T):
    x, w, _, _ = inputs(T, 600, 20, torch.float32)
    tiny = 2.0 ** -140
    x.zero_()
    x[:, 3], x[:, 599] = tiny, 1.0
    w[:, 3], w[:, 599] = 2.0 ** 20, 0.0
    assert (api.sp_linear(x, w) == 2.0 ** -120).all()                # exact: one product, its sum in fp64
    w[5, 599], w[6, 599], w[7, 3] = math.inf, -math.inf, math.nan
    y = api.sp_linear(x, w)
    assert (y[:, 5] == math.inf).all() and (y[:, 6] == -math.inf).all() and torch.isnan(y[:, 7]).all()
    assert (y[:, :5] == 2.0 ** -120).all() and (y[:, 8:] == 2.0 ** -120).all()


@pytest.mark.parametrize("T", [1, 20, 600])
def test_captured_calls_in_fp32(T):
    x, w, o, b = inputs(T, 300, 90, torch.float32)
    want = check(x, w, bias=b, act=api.SP_LINEAR_RELU, other=o)
    out = torch.zeros(T, 90, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.sp_linear(x, w, bias=b, act=api.SP_LINEAR_RELU, other=o, out=out)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("T,K,N", [(33, 768, 1536), (64, 1000, 4096), (65, 64, 4033), (192, 333, 1365), (192, 64, 1366), (193, 777, 100)])
def test_bf16_on_both_sides_of_the_choice_of_form(T, K, N):
    x, w, o, b = inputs(T, K, N, torch.bfloat16, seed=N)
    check(x, w)
    check(x, w, bias=b, act=api.SP_LINEAR_SILU, other=o, combine=api.SP_COMBINE_MUL)
    y = check(x, w, bias=b, act=api.SP_LINEAR_GELU, out_dtype=torch.float32)
    assert y.dtype == torch.float32


@pytest.mark.parametrize("dtype", DTYPES)
def test_tiles_of_many_rows(dtype):
    """What the tests above ask of few rows, of the general forms: in place, odd pitches, what stands beside ragged rows."""
    test_other_in_place(dtype, 600, api.SP_COMBINE_ADD)
    test_other_in_place(dtype, 600, api.SP_COMBINE_MUL)
    test_pitches_and_what_lies_beside_the_result(dtype, 600)
    test_values_beside_a_ragged_width_do_not_enter(dtype, 600)
    test_fp32_result_of_bf16_operands(api.SP_LINEAR_GELU, 600)
    test_infinities_and_nan(600)
