"""Values and batches at the edges of the operators: rows of few numbers, logits far from zero, logits beyond fp32, sequences of very
different lengths in one call."""
import math

import pytest
import torch

from paper_2510_03246_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]


def best(x, n):
    """Indices of the n best logits of every row: falling, the lower index first, NaN behind all."""
    y = torch.where(torch.isnan(x), -math.inf, x.double())
    order = torch.sort(y, dim=1, descending=True, stable=True).indices
    nan = torch.isnan(x).gather(1, order)
    return order.gather(1, torch.sort(nan.int(), dim=1, stable=True).indices)[:, :n]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_alts", [1, 8, 32])
@pytest.mark.parametrize("V", [40, 600, 4097, 9001, 70001])
def test_alternatives_of_rows_of_few_numbers(dtype, V, n_alts):
    """Rows of NaN but for some: every place is written, NaN behind all numbers and in the order of their indices."""
    x = torch.full((9, V), math.nan, dtype=dtype, device=DEV)
    x[1, V // 2] = 3.0
    x[2, [V - 1, 5, V // 3]] = torch.tensor([1.0, 1.0, -2.0], dtype=dtype, device=DEV)
    x[3, 7:20] = -math.inf
    x[4, ::2] = 0.5
    x[5, 1:] = -math.inf
    x[6] = -math.inf
    x[6, V // 4] = math.nan
    x[7] = torch.randn(V, device=DEV).to(dtype)
    x[7, ::3] = math.nan
    x[8, 11] = math.inf
    ids = torch.full((9, n_alts), -7, dtype=torch.int32, device=DEV)
    alt = torch.full((9, n_alts), 7.0, device=DEV)
    m = api.mat(x)
    assert api.lib().sp_token_logprobs(api.C.byref(m), None, 1.0, n_alts, None, None, None, ids.data_ptr(), alt.data_ptr(), None,
                                       torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(ids.long(), best(x, n_alts))
    assert torch.isnan(alt).all()                                  # a row with a NaN has no log probabilities
