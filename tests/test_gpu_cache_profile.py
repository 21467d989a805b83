"""What the kernels of sp_cache_attention are booked as."""
import pytest
import torch

from paper_2510_03246_b200 import api
from tests.test_gpu_paged_cache import filled, gen, ints, offsets, table_for

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("four", [False, True])
def test_what_a_cache_s_kernels_are_booked_as(four):
    """Products of the tensor cores, few rows or many; opening pages by itself."""
    heads, kv, dh, page = 8, 2, 64, 16
    for q_len, k_len, kinds in (([1, 2], [300, 40], {"gemm_tc": 1}), ([300], [900], {"gemm_tc": 1, "elementwise": 1})):
        table, n_pages = table_for(k_len, page, 74)
        pages = filled(n_pages, kv, page, dh, four, 75)
        Q = torch.randn(sum(q_len), heads * dh, generator=gen(76), device=DEV).to(BF)
        api.sp_profile_begin(1)
        try:
            api.sp_cache_attention(Q, pages, ints(offsets(q_len)), table, ints(k_len), heads)
            torch.cuda.synchronize()
            got = {k: v["records"] for k, v in api.sp_profile_read().items() if v["records"]}
        finally:
            api.sp_profile_begin(0)
        assert got == kinds
