"""Attention over contexts whose positions times the query heads of a group pass 32 bits."""
import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from paper_2608_13076_gb300 import int4

pytestmark = pytest.mark.gpu

SLICE = 64  # slots of a page


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


def halves(n, dev):
    """A block table for n slots in pages of 64: pages 0 .. 3 in turn for the first three quarters, then 4 .. 7."""
    pages = n // SLICE
    t = torch.arange(pages, dtype=torch.int32, device=dev) % 4
    t[3 * pages // 4:] += 4
    return t[None].contiguous()


@pytest.mark.parametrize("cache", ["bf16", "int4"])
def test_attention_far_positions(dev, cache):
    """50 million slots under 64 query heads: every key scores 0 and the values are 1, then -1, so that the output is the
    difference of their shares; sums of so many equal terms are exact in fp32."""
    n, D, Hq, k = 50 * 10**6 // 256 * 256, 64, 64, 2
    ctx = torch.tensor([n - 1 - k], dtype=torch.int32, device=dev)
    kd, cu = torch.tensor([k], dtype=torch.int32, device=dev), torch.tensor([0, k + 1], dtype=torch.int32, device=dev)
    q = torch.randn((k + 1, Hq, D), device=dev, generator=torch.Generator(device=dev).manual_seed(66)).to(torch.bfloat16)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((k + 1, Hq), float("nan"), dtype=torch.float32, device=dev)
    ws = spade.attn_workspace(1, Hq, 1, D, n, k, device=dev)
    st = spade.status_tensor(dev)
    table = halves(n, dev)
    if cache == "bf16":
        keys = torch.zeros((8, 1, SLICE, D), dtype=torch.bfloat16, device=dev)
        vals = torch.ones_like(keys)
        vals[4:] = -1
        spade.spade_verify_attention_paged(q, keys, vals, table, ctx, kd, cu, out, lse, max_k=k, workspace=ws, status=st)
    else:
        kc, kp, vc, vp = int4.kv4_pools(8, 1, SLICE, D, device=dev)
        vp[..., 0] = 1
        vc[:4] = 0x11   # code 1, zero 0
        vp[4:, ..., 1] = 1  # code 0, zero 1
        spade.spade_verify_attention_kv4(q, kc, kp, vc, vp, table, ctx, kd, cu, out, lse, max_k=k, workspace=ws, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for i in range(k + 1):
        seen, ones = n - k + i, 3 * n // 4
        want = (2 * ones - seen) / seen
        assert (out[i].double() - want).abs().max() <= 2.0 ** -8 * abs(want)
        # log2 of 2^7 times the count, near 33: an ulp of 2^-18, and half ulps of the sum and product after it.
        assert (lse[i].double() - np.log(seen)).abs().max() <= 2.0 ** -17
