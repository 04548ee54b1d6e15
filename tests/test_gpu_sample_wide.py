"""spade_sample on logits whose differences pass fp32's range or lie at its lower end, at temperatures of that size."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_sample import call, check, uniforms

pytestmark = pytest.mark.gpu
DEV = "cuda"
OPTIONS = [dict(), dict(top_k=700), dict(top_p=0.8), dict(min_p=0.05), dict(top_k=3000, top_p=0.9), dict(min_p=0.01, top_p=0.7)]


@pytest.mark.parametrize("opts", OPTIONS, ids=str)
@pytest.mark.parametrize("temperature", [1e38, 3.4e38, 2.0 ** 64, 1.5 * 2.0 ** 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [900, 32003])
def test_logits_as_far_apart_as_their_type_allows(gpu_lib, V, dtype, temperature, opts):
    """Differences of up to twice the largest finite number, whose weights are e^-6 at a temperature of 1e38; and of some
    temperatures, where the largest and the smallest are not that far."""
    gen = torch.Generator().manual_seed(V)
    part = torch.rand((4, V), generator=gen, dtype=torch.float64) * 2 - 1
    size = torch.tensor([3.3e38, 1e38, 2e38, 3.3e38], dtype=torch.float64)[:, None]
    x = part * torch.minimum(size, torch.tensor(8.0 * temperature, dtype=torch.float64))
    x[3, 5:] = -3.3e38
    x[3, 0], x[3, 4] = 3.3e38, 0.0
    x = x.to(dtype).to(DEV)
    u = uniforms(4, V + 1)
    t = float(np.float32(temperature))
    for probs in (True, False):
        tok, pr, ch, st = call(gpu_lib, x, u, temperature=t, probs=probs, **opts)
        assert st == 0
        check(x, u, tok, pr, ch, temperature=t, loose=2.0 ** -21 if probs else 2.0 ** -20 + 2.0 ** -21, **opts)


@pytest.mark.parametrize("probs", [True, False])
def test_a_uniform_beside_an_edge_at_a_huge_temperature(gpu_lib, probs):
    """Weights to 2^-39 there too: 30000 equal tokens behind one whose logit differs by a few thousandths of the
    temperature.  The first token's end lies 2^-24 Z or more from u Z, and 2^-33 of a weight matters nowhere else."""
    V, t = 32000, float(np.float32(2.5e38))
    x = torch.full((1, V), -1e38, dtype=torch.float32, device=DEV)
    x[0, V // 2:] = 1e38
    w = math.exp((float(np.float32(-1e38)) - float(np.float32(1e38))) / t)
    first = V // 2 * w / (V // 2 * (1 + w))   # the mass of the lower half
    for shift in (-3, -2, 2, 3):
        u = np.float32(first) + np.float32(shift * 2.0 ** -25)
        mass = float(u) * (1 + w)
        want = int(mass / w * (V // 2)) if mass < w else V // 2 + int((mass - w) * (V // 2))
        tok, _, _, st = call(gpu_lib, x, u, temperature=t, probs=probs)
        assert st == 0 and int(tok[0]) == want


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 1.2e-38])
@pytest.mark.parametrize("opts", [dict(), dict(top_p=0.7), dict(top_p=0.99999), dict(top_k=9), dict(min_p=0.3)], ids=str)
@pytest.mark.parametrize("V", [900, 32003])
def test_the_smallest_temperatures(gpu_lib, V, temperature, opts):
    """Down to where log2(e) / T is no finite number: equal largest logits share the mass, all others have none."""
    gen = torch.Generator().manual_seed(V)
    x = torch.randn((4, V), generator=gen)
    x[1, ::7] = x[1].max()
    x[2] = 1.5
    x[3, 5] = x[3].max() * (1 + 2.0 ** -20)
    x, u, t = x.to(DEV), uniforms(4, V + 2), float(np.float32(temperature))
    for probs in (True, False):
        tok, pr, ch, st = call(gpu_lib, x, u, temperature=t, probs=probs, **opts)
        assert st == 0
        check(x, u, tok, pr, ch, temperature=t, loose=2.0 ** -21 if probs else 2.0 ** -20 + 2.0 ** -21, **opts)
