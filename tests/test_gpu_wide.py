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


@pytest.mark.parametrize("R", [1, 9])
def test_projection_of_nearly_2_31_columns(dev, R):
    """The most columns that an int32 holds in whole groups: the first, a middle and the last one count, the
    others are zeros (an exact sum, worked by hand)."""
    K = 2**31 - 64
    x = torch.zeros((R, K), dtype=torch.bfloat16, device=dev)
    for at, v in ((0, 1.0), (K // 2 + 5, 2.0), (K - 1, 4.0)):
        x[:, at] = v
    codes = torch.full((1, K // 2), 0x33, dtype=torch.uint8, device=dev)  # 3 - 1 everywhere
    params = torch.ones((1, K // 64, 2), dtype=torch.float16, device=dev)
    out, st = torch.zeros((R, 1), dtype=torch.bfloat16, device=dev), spade.status_tensor(dev)
    spade.spade_linear_w4(x, codes, params, out, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and (out == 14).all()
