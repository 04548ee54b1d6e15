"""The 4-bit attention's outputs where one key takes all the weight, for scores of any size."""
import numpy as np
import pytest
import torch

from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4
from tests import int4_cases as C
from tests.test_gpu_kv4_long import big_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("up,scale", [(0, 1.0), (8, 0.125), (60, 4096.0), (-4, 64.0)])
def test_attention_one_key_takes_all(dev, D, up, scale):
    """One key of every (sequence, KV head) is aligned with the queries, every other one is not: the output is that
    slot's value.  Queries are +-2^up and keys whole numbers times a power of two, so scores are exact sums in fp32, the
    next one far below (its weight is taken from the numbers themselves).  What is left: the value in float16 (2^-11),
    fp32 quotients (2^-18) and bf16 (2^-8); of the lse a few fp32 products (2^-20)."""
    Hkv, G, page = 3, 4, 64
    unit = 2.0 ** up * scale
    c = big_cache(dev, [0, 5, 127, 128, 700, 3000], [3, 0, 8, 2, 4, 8], Hkv, D, page, 64)
    gen = torch.Generator().manual_seed(65)
    c["pools"][1][..., 0] = torch.where(c["pools"][1][..., 0].isnan(), float("nan"), scale).half()
    c["pools"][1][..., 1] = 8.0
    sign = torch.where(torch.rand((c["B"], Hkv, D), generator=gen) < 0.5, -1.0, 1.0)
    q = torch.empty((c["R"], Hkv * G, D))
    want = torch.empty((c["R"], Hkv * G, D), dtype=torch.float64)
    codes = int4.unpack_codes(c["pools"][0].cpu())
    table = c["table"].cpu().long()
    pools = [C.np64(t) for t in c["pools"]]
    for b in range(c["B"]):
        rows = slice(int(c["cu"][b]), int(c["cu"][b + 1]))
        for h in range(Hkv):
            s = [int(c["ctx"][b]), 0, int(c["ctx"][b]) // 2][h]  # the last slot that every row sees, the first, a middle one
            s = min(s, int(c["ctx"][b]))
            codes[table[b, s // page], h, s % page] = torch.where(sign[b, h] > 0, 15, 0).to(codes.dtype)
            q[rows, h * G:(h + 1) * G] = sign[b, h] * 2.0 ** up
            at = int(table[b, s // page]), h, s % page
            want[rows, h * G:(h + 1) * G] = torch.from_numpy(O.values(pools[2][at][None], pools[3][at][None])[0])
    c["pools"][0].copy_(int4.pack_codes(codes))
    q = q.to(torch.bfloat16).to(dev)
    tops = {}
    for b in range(c["B"]):
        n = int(c["ctx"][b] + c["k"][b]) + 1
        for h in range(Hkv):
            K = codes[table[b], h].reshape(-1, D)[:n].double() - 8
            s = (K @ sign[b, h].double()).sort().values
            assert float(s[-1] - s[-2]) * unit / D ** 0.5 >= 16
            rows = slice(int(c["cu"][b]), int(c["cu"][b + 1]))
            tops[b, h] = rows, float(s[-1]) * unit / D ** 0.5, float(s[-1] - s[-2]) * unit / D ** 0.5
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for (b, h), (rows, top, gap) in tops.items():
        hq = slice(h * G, (h + 1) * G)
        v, got = want[rows, hq], out[rows, hq].double().cpu()
        others = (int(c["ctx"][b] + c["k"][b]) + 1) * np.exp(-min(gap, 700.0)) * 8  # weights times values of size 8 at most
        assert ((got - v).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18) * v.abs() + others + 2.0 ** -24).all(), (b, h)
        assert ((lse[rows, hq].double().cpu() - top).abs() <= 2.0 ** -20 * (1 + abs(top)) + others).all(), (b, h)
