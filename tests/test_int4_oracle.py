"""The comparison of cached numbers sees scales and zeros that are not numbers (CPU)."""
import numpy as np
import pytest
import torch

from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4


def _case():
    x = torch.randn((8, 128), generator=torch.Generator().manual_seed(6))
    codes, params = int4.quantize(x, 64)
    return x.double().numpy(), codes, params.float()


def test_it_passes():
    x, codes, params = _case()
    assert O.check_quantised(x, np.zeros(x.shape), codes.numpy(), params.numpy()) == 0


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), -1.0])
@pytest.mark.parametrize("zeroed", [False, True])
def test_a_wrong_pair_is_seen(which, value, zeroed):
    """Also where the group's codes and zero are those of an empty one."""
    x, codes, params = _case()
    if zeroed:
        codes[2, 32:] = 0
        params[2, 1] = 0
    params[2, 1, which] = value
    assert O.check_quantised(x, np.zeros(x.shape), codes.numpy(), params.numpy()) > 0


def test_poisoned_cache_is_seen():
    x, codes, params = _case()
    params[..., 0], params[..., 1] = float("nan"), 0
    assert O.check_quantised(x, np.zeros(x.shape), torch.zeros_like(codes).numpy(), params.numpy()) >= 16


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_groups_that_are_not_finite(bad):
    """Such a group has to be poisoned, the one beside it must not be."""
    x, *_ = _case()
    x[3, 70] = bad
    codes, params = int4.quantize(torch.from_numpy(x).float(), 64)
    assert O.check_quantised(x.astype(np.float32).astype(np.float64), np.zeros(x.shape), codes.numpy(),
                             params.float().numpy()) == 0
    clean = params.clone()
    clean[3, 1, 0] = 1.0
    assert O.check_quantised(x, np.zeros(x.shape), codes.numpy(), clean.float().numpy()) > 0
