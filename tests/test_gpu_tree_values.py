"""spade_verify_attention_tree where values of the block are not finite: what reaches the outputs of rows that see them."""
import pytest
import torch

from tests import tree_cases as T

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("D,ctx,k,G,page", [(128, [150, 30], [40, 6], 4, 0), (64, [20_000], [40], 1, 64), (128, [1500], [200], 2, 0),
                                           (64, [0, 700], [127, 127], 2, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_the_lse_of_rows_that_see_a_value_that_is_not_finite(gpu_lib, D, ctx, k, G, page, bad):
    """Such a row is NaN in every dim; its lse is the scores' alone."""
    c = T.cache(ctx, k, 2, D, page, 151, DEV)
    q = T.queries(c, G, 152)
    mask = T.tree_mask(T.parents(k, "tree", 153), k, c["cu"].cpu())
    out, lse, st = T.attention(c, q, mask)
    for node in (3, k[-1]):
        slot = ctx[-1] + node
        if page:
            c["v"][c["table"][-1, slot // page], 1, slot % page, 5] = bad
        else:
            c["v"][-1, 1, slot, 5] = bad
    again, l2, st2 = T.attention(c, q, mask)
    assert int(st.item()) == int(st2.item()) == 0
    assert torch.equal(lse, l2) and bool(l2.isfinite().all())
    r0 = int(c["cu"][-2])
    sees = torch.zeros(c["R"], dtype=torch.bool)
    for node in (3, k[-1]):
        sees[r0:] |= (mask[r0:, node // 32] >> (node % 32) & 1).bool()
    assert bool(again[sees][:, G:].isnan().all())
    assert torch.equal(again[~sees], out[~sees]) and torch.equal(again[:, :G], out[:, :G])


def test_scores_that_are_not_finite(gpu_lib):
    """A key that is NaN makes the rows that see it NaN, their lse too."""
    c = T.cache([300], [20], 1, 128, 0, 161, DEV)
    q = T.queries(c, 2, 162)
    mask = T.tree_mask(T.parents([20], "tree", 163), [20], c["cu"].cpu())
    c["k"][0, 0, 300 + 4, 9] = float("nan")
    c["v"][0, 0, 300 + 4, 9] = float("nan")
    out, lse, st = T.attention(c, q, mask)
    sees = (mask[:, 0] >> 4 & 1).bool()
    assert int(st.item()) == 0
    assert bool(out[sees].isnan().all()) and bool(lse[sees].isnan().all())
    assert bool(out[~sees].isfinite().all()) and bool(lse[~sees].isfinite().all())
