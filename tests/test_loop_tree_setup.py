"""What the tree loop's verifier keeps and sets up (CPU: no kernel is launched)."""
import torch

from paper_2608_13076_gb300 import rope
from paper_2608_13076_gb300 import speculative as S


def test_one_workspace_for_prompts_of_all_lengths(monkeypatch):
    """A verifier that has met many lengths of prompts and blocks holds one workspace of the attention."""
    made = []
    monkeypatch.setattr(S, "tree_attn_workspace", lambda *a, **k: made.append(torch.zeros(8)) or made[-1])
    used = []
    monkeypatch.setattr(S, "spade_tree_layout", lambda *a, **k: None)
    monkeypatch.setattr(S, "spade_verify_rope_paged", lambda *a, **k: None)
    monkeypatch.setattr(S, "spade_verify_attention_tree_paged", lambda *a, workspace, **k: used.append(workspace))
    v = S.ToyVerifierTree(S.ToyConfig(), 1, 100, seed=1, device="cpu")
    for n in (3, 9, 40, 41, 77):
        kd, cu = torch.tensor([n - 1], dtype=torch.int32), torch.tensor([0, n], dtype=torch.int32)
        v.write_prefix(torch.arange(n), v.ctx, kd, cu, n - 1)
    assert len(made) == 1 and len(used) == 5 * v.layers and all(w is made[0] for w in used)


def test_stretched_frequencies_bring_no_factor_of_their_own():
    """A model with stretched bands has a factor on its turned dims where it is given one, and none otherwise."""
    scaling = dict(kind="bands", factor=8.0, context=64)
    v = S.ToyVerifierTree(S.ToyConfig(), 1, 64, seed=1, device="cpu", scaling=scaling)
    assert v.mscale == 1.0
    w = S.ToyVerifierTree(S.ToyConfig(), 1, 64, seed=1, device="cpu", scaling=scaling, mscale=rope.attention_scale(8.0))
    assert w.mscale == rope.attention_scale(8.0) and torch.equal(v.inv_freq, w.inv_freq)
