"""spade_sample where its sums have to be exact: rows whose tails are far below the largest weight, with uniforms and
bounds just beside an edge.  Rows are a few groups of equal logits, so that edges are known as fractions."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from tests.test_gpu_sample import call

pytestmark = pytest.mark.gpu
DEV = "cuda"
# Weights are known to 2^-39 of the largest, so a cumulative mass is known to a few of those where few weights are large.
SURE = Fraction(1, 2 ** 37)


def row_of(V, dtype, groups):
    """[1, V] of runs (count, logit); a count of None takes the rest."""
    rest = V - sum(n for n, _ in groups if n is not None)
    runs = [(rest if n is None else n, torch.tensor(x, dtype=torch.float64).to(dtype)) for n, x in groups]
    return torch.cat([x.expand(n) for n, x in runs])[None].to(DEV), [(n, float(x)) for n, x in runs]


def mass_of(runs, temperature=1.0):
    top = max(x for _, x in runs)
    return [n * Fraction(math.exp((x - top) / temperature)) for n, x in runs]


def run_of(runs, u):
    """(index of the run in which cumulative mass passes u of the whole, how far that is from the run's ends)."""
    mass = mass_of(runs)
    goal, at = Fraction(float(np.float32(u))) * sum(mass), Fraction(0)
    for i, m in enumerate(mass):
        if at + m > goal:
            return i, min(goal - at if i else goal, at + m - goal)
        at += m
    raise AssertionError


def check_draw(lib, V, dtype, groups, u, probs, **opts):
    x, runs = row_of(V, dtype, groups)
    want, near = run_of(runs, u)
    assert near > SURE, (float(near), want)
    tok, pr, ch, st = call(lib, x, u, probs=probs, **opts)
    first = np.cumsum([0] + [n for n, _ in runs])
    assert st == 0
    assert first[want] <= int(tok[0]) < first[want + 1], (int(tok[0]), want, first.tolist(), float(near))
    return runs, want


TYPES = [(torch.float32, 128256), (torch.bfloat16, 128256), (torch.float16, 128256), (torch.bfloat16, 1_500_000),
         (torch.float32, 700_001), (torch.float16, 1_500_001)]


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("u", [0.5 + 2.0 ** -24, 0.5 + 2.0 ** -23])
@pytest.mark.parametrize("dtype,V", TYPES)
def test_a_tail_of_nothing_between_two_tokens(gpu_lib, dtype, V, u, probs):
    """0 at the first and the last token, -100 between: the last is drawn, not a token of probability e^-100."""
    check_draw(gpu_lib, V, dtype, [(1, 0.0), (None, -100.0), (1, 0.0)], u, probs)


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("dtype,V", TYPES)
def test_a_token_beside_the_middle(gpu_lib, dtype, V, probs):
    """Weights 1, a tail of e^-100, 1, e^-21: half the mass lies 2^-32 behind the tail."""
    check_draw(gpu_lib, V, dtype, [(1, 0.0), (None, -100.0), (1, 0.0), (1, -21.0)], 0.5, probs)


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("tail", [-32.0, -45.0, -100.0, -700.0])
@pytest.mark.parametrize("near", [30, 32, 34, 35])
@pytest.mark.parametrize("dtype,V", TYPES)
def test_uniforms_beside_an_edge(gpu_lib, dtype, V, near, tail, probs):
    """Half the mass lies 2^-near on either side of the tail's end (a last token weighs a little more or less than the
    tail), or before its beginning."""
    t = (V - 3) * math.exp(tail)
    weights = [t + 2.0 ** (1 - near)] + ([t - 2.0 ** (1 - near)] if t > 2.0 ** (1 - near) else [])
    for w in weights:
        check_draw(gpu_lib, V, dtype, [(1, 0.0), (None, tail), (1, 0.0), (1, math.log(w))], 0.5, probs)
    if dtype is not torch.float16:  # whose numbers are not that small
        check_draw(gpu_lib, V, dtype, [(1, 0.0), (None, tail), (1, -t - 2.0 ** (1 - near))], 0.5, probs)


@pytest.mark.parametrize("near", [30, 33, 35])
@pytest.mark.parametrize("dtype,V", TYPES[:2] + TYPES[3:5])
def test_two_thousand_listed_tokens(gpu_lib, dtype, V, near):
    """The same where the tail is a list that one CTA decides on: two thousand tokens that min_p keeps."""
    n = 2000
    x, runs = row_of(n + 2, dtype, [(1, 0.0), (n, -100.0), (1, -2.0 ** (1 - near))])
    want, off = run_of(runs, 0.5)
    assert want == 0 and off > SURE
    wide = torch.full((1, V), -110.0, dtype=dtype, device=DEV)
    wide[0, ::V // (n + 2)][:n + 2] = x[0]
    for probs in (False, True):
        tok, pr, ch, st = call(gpu_lib, wide, 0.5, min_p=1e-44, probs=probs)
        assert st == 0 and int(tok[0]) == 0
        if probs:
            assert int((pr > 0).sum()) == n + 2


@pytest.mark.parametrize("near", [31, 33, 35])
@pytest.mark.parametrize("tail", [-32.0, -100.0])
@pytest.mark.parametrize("dtype,V", TYPES[:2] + TYPES[3:5])
def test_a_nucleus_that_ends_beside_a_token(gpu_lib, dtype, V, near, tail):
    """Two tokens nearly alike and a tail: the first has half the mass, or 2^-near less than that."""
    t = (V - 2) * math.exp(tail)
    for less in [t + 2.0 ** (1 - near)] + ([t - 2.0 ** (1 - near)] if t > 2.0 ** (1 - near) else []):
        x, runs = row_of(V, dtype, [(1, 0.0), (None, tail), (1, -less)])
        mass = mass_of(runs)
        off = mass[0] - sum(mass) / 2
        assert abs(off) > SURE
        tok, pr, ch, st = call(gpu_lib, x, 0.25, top_p=0.5)
        assert st == 0 and int((pr > 0).sum()) == (1 if off > 0 else 2) and int(tok[0]) == 0


@pytest.mark.parametrize("tail", [-45.0, -100.0])
@pytest.mark.parametrize("top_p", [0.99985, 0.9999, 0.99995, 0.99999, 1 - 2.0 ** -18])
def test_a_nucleus_of_many_tokens(gpu_lib, top_p, tail):
    """One token, a hundred thousand of e^-20 each, different all, and a tail: the nucleus ends among the many."""
    V, n = 128256, 100_000
    many = (-20.0 - np.arange(n) * 2.0 ** -18).astype(np.float32)
    x = np.full(V, tail, dtype=np.float32)
    x[0] = 0.0
    place = 1 + np.random.RandomState(1).permutation(V - 1)[:n]
    x[place] = many
    w = np.exp(many.astype(np.float64))
    behind = np.cumsum(w)  # beside the first token's 1: errors of n 2^-53 of 2^-12
    p = Fraction(float(np.float32(top_p)))
    goal = float(p * (1 + Fraction(float(behind[-1])) + (V - 1 - n) * Fraction(math.exp(tail))) - 1)
    want = int(np.searchsorted(behind, goal))
    assert 0 < want < n and np.abs(behind - goal).min() > 2.0 ** -38, (want, np.abs(behind - goal).min())
    for probs in (True, False):
        tok, pr, ch, st = call(gpu_lib, torch.from_numpy(x)[None].to(DEV), 0.0, top_p=top_p, probs=probs)
        assert st == 0 and int(tok[0]) == 0
        if probs:
            assert int((pr > 0).sum()) == want + 2
            assert bool((pr[0, torch.from_numpy(place[:want + 1]).to(DEV)] > 0).all())
        kept = 1 + float(behind[want])
        assert abs(float(ch[0]) - 1 / kept) <= 2.0 ** -20
