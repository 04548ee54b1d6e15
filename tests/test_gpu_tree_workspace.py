"""One workspace of the tree attention for calls of many sizes."""
import pytest
import torch

from tests import tree_cases as T

pytestmark = pytest.mark.gpu
DEV = "cuda"

# ctx, k, G, Hkv, D, page: units split over CTAs, with few and many units, row groups and parts, both head dims
SIZES = [
    ([4000] * 8, [511] * 8, 4, 8, 128, 0),
    ([4000] * 8, [63] * 8, 4, 8, 128, 0),
    ([30_000], [5], 4, 1, 64, 64),
    ([3000, 200], [300, 2], 1, 2, 64, 0),
    ([9000], [130], 8, 1, 128, 128),
    ([100] * 30, [3] * 30, 2, 4, 64, 64),
]


def test_one_workspace_for_calls_of_all_sizes(gpu_lib):
    """The same bits as with workspaces of their own, in every order of sizes."""
    calls, need = [], 0
    for i, (ctx, k, G, Hkv, D, page) in enumerate(SIZES):
        c = T.cache(ctx, k, Hkv, D, page, 200 + i, DEV)
        q = T.queries(c, G, 300 + i)
        mask = T.tree_mask(T.parents(k, "tree", 400 + i), k, c["cu"].cpu()).to(DEV)
        out, lse, st = T.attention(c, q, mask)
        assert int(st.item()) == 0 and bool(out.isfinite().all())
        need = max(need, gpu_lib.spade_tree_attn_workspace_size(c["B"], G * Hkv, Hkv, D, c["cap"], c["max_k"]))
        calls.append((c, q, mask, out, lse))
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    n = len(calls)
    for a in range(n):
        for b in range(n):
            for i in (a, b):
                c, q, mask, out, lse = calls[i]
                got, l, st = T.attention(c, q, mask, workspace=ws)
                assert int(st.item()) == 0
                assert torch.equal(got, out) and torch.equal(l, lse), (a, b, i)


def test_the_size_depends_on_the_head_dim_alone(gpu_lib):
    """So a program keeps one workspace, whatever the sizes of its calls."""
    for D in (64, 128):
        sizes = {gpu_lib.spade_tree_attn_workspace_size(B, G * Hkv, Hkv, D, cap, k) for B, G, Hkv, cap, k in
                 ((1, 1, 1, 64, 0), (8, 4, 8, 4608, 511), (512, 8, 8, 1024, 100), (3, 5, 2, 40_000, 2000))}
        assert len(sizes) == 1



@pytest.mark.parametrize("ctx,k,G,Hkv,D", [([30_000], [5], 4, 1, 128), ([3000, 200], [300, 2], 1, 2, 64)])
def test_only_the_counters_have_to_be_zero(gpu_lib, ctx, k, G, Hkv, D):
    """What lies behind them in a new workspace does not matter."""
    c = T.cache(ctx, k, Hkv, D, 0, 210, DEV)
    q = T.queries(c, G, 211)
    mask = T.tree_mask(T.parents(k, "tree", 212), k, c["cu"].cpu())
    out, lse, st = T.attention(c, q, mask)
    ws = torch.full_like(gpu_lib.tree_attn_workspace(c["B"], G * Hkv, Hkv, D, c["cap"], c["max_k"]), 255)
    ws[:gpu_lib.TREE_ATTN_ZEROED] = 0
    got, l2, st2 = T.attention(c, q, mask, workspace=ws)
    assert int(st.item()) == int(st2.item()) == 0
    assert torch.equal(got, out) and torch.equal(l2, lse)
