"""Sizes that 32 bits do not hold are refused by the Python entry points, not cut."""
import pytest
import torch

import paper_2608_13076_gb300 as spade
from tests import int4_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


def test_columns_past_32_bits(dev):
    K = 2**32 + 64
    x = torch.empty((1, K), dtype=torch.bfloat16, device=dev)
    codes = torch.empty((1, K // 2), dtype=torch.uint8, device=dev)
    params = torch.empty((1, K // 64, 2), dtype=torch.float16, device=dev)
    out, st = torch.zeros((1, 1), dtype=torch.bfloat16, device=dev), spade.status_tensor(dev)
    with pytest.raises(ValueError, match="2\\^31"):
        spade.spade_linear_w4(x, codes, params, out, status=st)


@pytest.mark.parametrize("max_k", [2**32 + 2, 2**31, -2**31 - 1, 2**64])
def test_bound_past_32_bits(dev, max_k):
    c = C.cache([100, 40], [2, 1], 2, 128, 64, 28, dev)
    q = C.queries(c, 2, 29)
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device=dev)
    with pytest.raises((ValueError, OverflowError)):
        C.attention(c, q, max_k=max_k, workspace=ws)
