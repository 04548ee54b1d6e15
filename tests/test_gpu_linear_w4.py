"""Projections with 4-bit weights on the GPU against float64: row counts, ragged sizes, every group size."""
import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4
from tests import int4_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


def _run(dev, R, N, K, group, residual, seed=1, scale=1.0, in_place=False):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((R, K), generator=g) * scale).to(torch.bfloat16)
    codes, params = int4.quantize(torch.randn((N, K), generator=g) / K ** 0.5, group)
    res = torch.randn((R, N), generator=g).to(torch.bfloat16) if residual else None
    st = spade.status_tensor(dev)
    out = torch.full((R + 2, N), float("nan"), dtype=torch.bfloat16, device=dev)
    given = None if res is None else res.to(dev)
    if in_place:
        out[:R] = given
        given = out[:R]
    spade.spade_linear_w4(x.to(dev), codes.to(dev), params.to(dev), out[:R], given, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and out[R:].isnan().all()
    return x, codes, params, res, out[:R]


def _check(x, codes, params, res, out):
    """Products of bf16 and whole numbers in 4 bits are exact in fp32; K of them are summed in fp32 (error at most
    K 2^-23 of the sum of their sizes), and the result is rounded to bf16 once (2^-8)."""
    r = None if res is None else C.np64(res).astype(np.float64)
    want, mass = O.linear(C.np64(x), codes.numpy(), params.numpy(), r)
    if r is not None:
        mass = mass + np.abs(r)
    tol = 2.0 ** -8 * np.abs(want) + x.shape[1] * 2.0 ** -23 * mass + 1e-38
    err = np.abs(C.np64(out).astype(np.float64) - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("R", [1, 2, 3, 7, 8, 9, 15, 16, 17, 24, 25, 31, 32, 33, 47, 48, 63, 64, 65, 72, 127, 128, 129])
def test_rows(dev, R, group, residual):
    _check(*_run(dev, R, 200, 384, group, residual))


@pytest.mark.parametrize("R", [1, 5, 20, 70, 300])
@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (1, 128, 128), (15, 64, 64), (16, 96, 32), (17, 1088, 64), (63, 160, 32),
                                       (65, 4096, 128), (127, 640, 128), (129, 2080, 32), (255, 192, 64), (257, 128, 64),
                                       (1000, 64, 32), (4421, 384, 128), (513, 8192, 64)])
def test_sizes(dev, R, N, K, group):
    _check(*_run(dev, R, N, K, group, N % 2 == 0))


@pytest.mark.parametrize("R,N,K,group", [(5, 20000, 4352, 32), (8, 19600, 2304, 64), (1, 40000, 512, 128), (3, 41, 4224, 128),
                                         (700, 5000, 1024, 128), (64, 39000, 256, 128), (200, 39000, 256, 64)])
def test_many_tiles(dev, R, N, K, group):
    """More outputs than one pass of the SMs holds sums for; tiles of outputs in pairs."""
    _check(*_run(dev, R, N, K, group, R % 2 == 0))


@pytest.mark.parametrize("R", [4, 40])
def test_residual_is_the_output(dev, R):
    _check(*_run(dev, R, 321, 256, 64, True, in_place=True))


@pytest.mark.parametrize("R", [4, 100])
@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_any_size_of_activations(dev, R, scale):
    _check(*_run(dev, R, 100, 512, 64, False, scale=scale))


@pytest.mark.parametrize("R", [3, 30, 100])
def test_not_finite(dev, R):
    """A NaN stays in its row; a poisoned group of weights in its column."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((R, 256), generator=g).to(torch.bfloat16).to(dev)
    codes, params = (t.to(dev) for t in int4.quantize(torch.randn((70, 256), generator=g), 64))
    st = spade.status_tensor(dev)
    clean, out = (torch.empty((R, 70), dtype=torch.bfloat16, device=dev) for _ in range(2))
    spade.spade_linear_w4(x, codes, params, clean, status=st)
    x[1, 200] = float("nan")
    params[33, 2, 0] = float("nan")
    spade.spade_linear_w4(x, codes, params, out, status=st)
    torch.cuda.synchronize()
    bad = torch.zeros((R, 70), dtype=torch.bool, device=dev)
    bad[1], bad[:, 33] = True, True
    assert torch.equal(out.isnan(), bad) and torch.equal(out[~bad], clean[~bad])


def test_largest_codes(dev):
    """Every code 15 over zero 0, and 0 over zero 15: the ends of the range, worked by hand."""
    for code, zero, v in ((255, 0.0, 15.0), (0, 15.0, -15.0)):
        codes = torch.full((40, 64), code, dtype=torch.uint8, device=dev)
        params = torch.tensor([0.5, zero], dtype=torch.float16).repeat(40, 2, 1).to(dev)
        for R in (2, 70):
            x, out = torch.ones((R, 128), dtype=torch.bfloat16, device=dev), torch.empty((R, 40), dtype=torch.bfloat16, device=dev)
            spade.spade_linear_w4(x, codes, params, out, status=spade.status_tensor(dev))
            assert (out == 128 * 0.5 * v).all()


def test_same_bits_again(dev):
    """Nothing depends on timing: repeated calls, and on another stream."""
    for R in (5, 90):
        *_, a = _run(dev, R, 700, 2048, 64, False)
        stream = torch.cuda.Stream(dev)
        for _ in range(3):
            with torch.cuda.stream(stream):
                *_, b = _run(dev, R, 700, 2048, 64, False)
            assert torch.equal(a, b)
