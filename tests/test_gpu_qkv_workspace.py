"""One workspace of the projection with rotary embedding for calls over layers of different widths."""
import pytest
import torch

import paper_2608_13076_gb300 as spade
from paper_2608_13076_gb300 import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"

# More rows than the kernel on pairs of CTAs takes, which needs no workspace; 48, 8 and 5 tiles.
SPECS = [
    W.WorkloadSpec("wide", B=52, Hq=32, Hkv=8, D=128, H=256, V=1000, ctx=(5, 60), k=(8, 8), mode="greedy", seed=71),
    W.WorkloadSpec("narrow", B=40, Hq=4, Hkv=2, D=128, H=256, V=1000, ctx=(5, 300), k=(6, 9), mode="greedy", seed=72),
    W.WorkloadSpec("d64", B=40, Hq=6, Hkv=2, D=64, H=520, V=1000, ctx=(5, 300), k=(6, 9), mode="greedy", seed=73),
]


def _call(wl, x, w, ws):
    st = spade.status_tensor(DEV)
    q = torch.full((wl["R"], wl["Hq"], wl["D"]), float("nan"), dtype=torch.bfloat16, device=DEV)
    k, v = wl["k_cache"].clone(), wl["v_cache"].clone()
    spade.spade_verify_qkv_rope(x, w, wl["ctx_lens"], wl["n_draft"], wl["cu_q"], q, k, v, Hq=wl["Hq"], Hkv=wl["Hkv"],
                                rope_theta=wl["spec"].rope_theta, max_k=int(wl["n_draft"].max()), workspace=ws, status=st)
    assert int(st.item()) == 0
    return q, k, v


def test_calls_of_all_widths_share_a_workspace(gpu_lib):
    """The bits of workspaces of their own, in every order."""
    calls, own, size = [], [], 0
    for spec in SPECS:
        wl = W.make_workload(spec, device=DEV)
        x, w = W.make_qkv_inputs(spec, wl["R"], device=DEV)
        calls.append((wl, x, w))
        ws = spade.qkv_workspace(wl["R"], wl["Hq"], wl["Hkv"], wl["D"], device=DEV)
        own.append(_call(wl, x, w, ws))
        size = max(size, ws.numel())
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    for a in range(len(calls)):
        for b in range(len(calls)):
            for i in (a, b):
                assert all(torch.equal(x, y) for x, y in zip(_call(*calls[i], ws), own[i])), (a, b, i)
