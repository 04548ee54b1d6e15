"""One attention workspace for calls of many sizes, of the bf16 caches and of the 4-bit one."""
import pytest
import torch

import paper_2608_13076_gb300 as spade
from tests import int4_cases as C
from tests import tree_cases as T

pytestmark = pytest.mark.gpu
DEV = "cuda"

# ctx, k, G, Hkv, D, page of the tree tests' caches (0: dense); units split over CTAs, many and few of them
SIZES = [
    ([1500] * 16, [40] * 16, 8, 8, 128, 0),
    ([1500] * 16, [3] * 16, 4, 8, 128, 0),
    ([9000], [5], 4, 1, 64, 64),
    ([2000, 200], [200, 2], 4, 2, 64, 0),
    ([100] * 30, [3] * 30, 2, 4, 128, 64),
]


def _bf16(c, q, workspace):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    st = spade.status_tensor(DEV)
    more = dict(max_k=c["max_k"], workspace=workspace, status=st)
    lens = (c["ctx"], c["n"], c["cu"])
    if c["page"]:
        spade.spade_verify_attention_paged(q, c["k"], c["v"], c["table"], *lens, out, lse, **more)
    else:
        spade.spade_verify_attention(q, c["k"], c["v"], *lens, out, lse, **more)
    return out, lse, st


def _share(calls, size, attend):
    """attend(call, workspace) -> (out, lse, status) of every pair of calls in a row, on one workspace: the bits of workspaces
    of their own."""
    own = [attend(c, torch.zeros(s, dtype=torch.uint8, device=DEV)) for c, s in zip(calls, size)]
    ws = torch.zeros(max(size), dtype=torch.uint8, device=DEV)
    for a in range(len(calls)):
        for b in range(len(calls)):
            for i in (a, b):
                out, lse, st = attend(calls[i], ws)
                assert int(st.item()) == int(own[i][2].item()) == 0
                assert torch.equal(out, own[i][0]) and torch.equal(lse, own[i][1]), (a, b, i)


def test_bf16_caches(gpu_lib):
    calls, size = [], []
    for i, (ctx, k, G, Hkv, D, page) in enumerate(SIZES):
        c = T.cache(ctx, k, Hkv, D, page, 500 + i, DEV)
        calls.append((c, T.queries(c, G, 600 + i)))
        size.append(spade.spade_attn_workspace_size(c["B"], G * Hkv, Hkv, D, c["cap"], c["max_k"]))
    _share(calls, size, lambda call, ws: _bf16(*call, ws))


def test_4_bit_cache(gpu_lib):
    calls, size = [], []
    for i, (ctx, k, G, Hkv, D, page) in enumerate(SIZES):
        c = C.cache(ctx, k, Hkv, D, 64, 700 + i, DEV)
        calls.append((c, C.queries(c, G, 800 + i)))
        size.append(spade.spade_attn_workspace_size(c["B"], G * Hkv, Hkv, D, c["max_pages"] * 64, c["max_k"]))
    _share(calls, size, lambda call, ws: C.attention(*call, workspace=ws))
