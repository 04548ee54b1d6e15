"""Algorithm 1 end to end with the verifier's projections and cache in 4 bits
(paper_2608_13076_gb300.speculative.ToyVerifierInt4)."""
import numpy as np
import pytest
import torch

from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4
from paper_2608_13076_gb300 import speculative as S
from tests import int4_cases as C

pytestmark = pytest.mark.gpu

B, MAX_NEW = 5, 30


@pytest.fixture(scope="module", params=[64, 128])
def verifier(request, gpu_lib):
    cfg = S.ToyConfig(D=request.param, Hq=512 // request.param, Hkv=2)
    return S.ToyVerifierInt4(cfg, B, cap=1024, seed=3, device="cuda:0", page=64 if request.param == 64 else 128,
                             group=64 if request.param == 64 else 128)


def _prompts(V, seed=4):
    g = np.random.default_rng(seed)
    return [list(g.integers(0, V - 1, size=int(n))) for n in (2, 70, 17, 128, 40)]


def test_greedy_speculative_equals_plain_decoding(verifier):
    """Greedy verification makes the output independent of the drafts (Sec. III-B): for every draft length the
    tokens are those of plain decoding with this verifier alone, but for near ties (top-2 gap below 0.05, logits
    ~ N(0, 16)): the runs sum in different orders."""
    prompts = _prompts(verifier.cfg.V)
    ref = S.speculative_decode(verifier, prompts, d=0, max_new=MAX_NEW, record_margins=True)
    for d in (1, 4):
        res = S.speculative_decode(verifier, prompts, d=d, max_new=MAX_NEW)
        identical = 0
        for b in range(B):
            a, r = res.tokens[b], ref.tokens[b]
            i = next((j for j in range(min(len(a), len(r))) if a[j] != r[j]), None)
            if i is None:
                assert len(a) == len(r), (d, b)
                identical += 1
            else:
                assert ref.margins[b][i] < 0.05, (d, b, i, ref.margins[b][i])
        assert identical >= B - 1, (d, identical)
        assert sum(res.calls_per_seq) < sum(ref.calls_per_seq)
    assert int(verifier.status.item()) == 0


def test_stochastic_loop_runs_and_accepts(verifier):
    res = S.speculative_decode(verifier, _prompts(verifier.cfg.V, 5), d=4, max_new=MAX_NEW, mode=S.STOCHASTIC, seed=9,
                               temperature=0.9, top_p=0.95)
    assert all(1 <= len(t) <= MAX_NEW and all(0 <= x < verifier.cfg.V for x in t) for t in res.tokens)
    assert 0 < res.accepted < res.drafted


def test_cache_after_a_loop(verifier):
    """After a loop the committed slots of a sequence hold what a float64 run over its tokens puts there."""
    cfg, prompts = verifier.cfg, _prompts(verifier.cfg.V, 6)
    res = S.speculative_decode(verifier, prompts, d=3, max_new=12)
    pools, table = [C.np64(t) for t in verifier.pools], C.np64(verifier.table)
    rope, emb = C.np64(verifier.rope), C.np64(verifier.emb)
    for b in range(B):
        tokens = (prompts[b] + res.tokens[b])[:len(prompts[b]) + len(res.tokens[b]) - 1]
        tokens = tokens[:int(verifier.ctx[b])]
        y, _ = O.linear(emb[np.array(tokens)], C.np64(verifier.w_qkv[0]), C.np64(verifier.w_qkv[1]))
        y = torch.from_numpy(y).to(torch.bfloat16).float().numpy().reshape(len(tokens), -1, cfg.D)
        k = y[:, cfg.Hq:cfg.Hq + cfg.Hkv]
        want, _ = O.turned(k, np.ones(cfg.D), rope[:len(tokens)], 1e-6)
        got = O.values(O.slots(pools[0], table[b], 0, len(tokens)), O.slots(pools[1], table[b], 0, len(tokens)))
        step = np.repeat(O.slots(pools[1], table[b], 0, len(tokens))[..., 0].astype(np.float64), 64, axis=-1)
        # Half a step of the quantiser (a step at the cut ends), and bf16 inputs that may fall on the other side of a
        # rounding (2^-8 of a head's largest number).
        assert (np.abs(got - want) <= 1.01 * step + 2.0 ** -7 * np.abs(want).max(-1, keepdims=True)).all()
