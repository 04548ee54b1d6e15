"""The 4-bit cache's kernels in steady state: attention whose CTAs walk units of dozens of key chunks, prompts that
take the cache write's form for many rows, and read-backs of more rows than the grid covers at once."""
import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4
from tests import int4_cases as C
from tests.test_gpu_kv4 import _check_heads, _norm_rope

pytestmark = pytest.mark.gpu

SLICE = 64  # keys


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


def sms(dev):
    return torch.cuda.get_device_properties(dev).multi_processor_count


def big_cache(dev, ctx, k, Hkv, D, page, seed):
    """int4_cases.cache, filled on the GPU."""
    gen = torch.Generator(device=dev).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    ctx, k, cu = C.lengths(ctx, k)
    B, n = len(ctx), -(-int((ctx + k).max() + 1) // page)
    pages = B * n + 2
    table = torch.randperm(pages, generator=host)[:B * n].reshape(B, n)
    live = torch.zeros((pages, page), dtype=torch.bool)
    live[table.reshape(-1)] = (torch.arange(n * page) <= (ctx + k)[:, None]).reshape(B * n, page)
    pools = []
    for _ in range(2):
        codes, params = int4.quantize(torch.randn((pages, Hkv, page, D), generator=gen, device=dev), 64)
        params[~live[:, None].expand(-1, Hkv, -1).to(dev)] = float("nan")
        pools += [codes, params]
    return dict(pools=pools, table=table.to(torch.int32).to(dev), ctx=ctx.to(dev), k=k.to(dev), cu=cu.to(dev), B=B,
                R=int(cu[-1]), max_k=int(k.max()), Hkv=Hkv, D=D, page=page, max_pages=n)


def part(c, G, q, out, lse, seqs, heads):
    """The sequences `seqs` and KV heads `heads` of a case alone: (case, q, out, lse)."""
    table = c["table"][seqs].long()
    at = [r for b in seqs for r in range(int(c["cu"][b]), int(c["cu"][b + 1]))]
    hq = [h * G + g for h in heads for g in range(G)]
    d = dict(c, pools=[p[table.reshape(-1)][:, heads].contiguous() for p in c["pools"]], ctx=c["ctx"][seqs], k=c["k"][seqs],
             table=torch.arange(table.numel(), dtype=torch.int32).reshape(table.shape), B=len(seqs), Hkv=len(heads))
    d["cu"] = C.lengths(d["ctx"].tolist(), d["k"].tolist())[2]
    return d, q[at][:, hq], out[at][:, hq], lse[at][:, hq]


def walks_far(c, G, dev):
    """Every CTA's share is more than 24 chunks of 128 keys, and a whole unit passes 64 slices: the copy ring, the slots
    of scales and the buffers wrap many times, and the page lookups are refilled twice."""
    n = [int(x) for x in (c["ctx"] + c["k"] + 1).tolist()]
    blocks = [-(-G * (int(x) + 1) // 64) for x in c["k"].tolist()]
    assert sum(-(-a // SLICE) * r for a, r in zip(n, blocks)) * c["Hkv"] / sms(dev) > 48
    assert max(n) > 65 * SLICE


RAGGED = [0, 1, 63, 64, 5999, 6000, 4161, 4160]


def ragged(B, lo=4300, hi=6000):
    return RAGGED + [lo + i * (hi - lo) // (B - len(RAGGED)) for i in range(B - len(RAGGED))]


LONG = {
    "one_token": dict(ctx=ragged(64), k=[0] * 64, Hkv=8, G=5, D=128, page=64),
    "one_token_d64": dict(ctx=ragged(64), k=[0] * 64, Hkv=8, G=1, D=64, page=64),
    "rows_20": dict(ctx=ragged(40), k=[4] * 40, Hkv=8, G=4, D=128, page=192),
    "rows_36": dict(ctx=ragged(24), k=[8] * 20 + [0, 3, 8, 8], Hkv=8, G=4, D=128, page=256),
    "rows_36_d64": dict(ctx=ragged(24), k=[8] * 20 + [0, 3, 8, 8], Hkv=8, G=4, D=64, page=256),
    "rows_64": dict(ctx=ragged(24), k=[7] * 24, Hkv=8, G=8, D=128, page=128),
    "two_row_blocks": dict(ctx=ragged(24), k=[10] * 23 + [2], Hkv=4, G=8, D=128, page=64),
    "two_row_blocks_d64": dict(ctx=ragged(24), k=[10] * 23 + [2], Hkv=4, G=8, D=64, page=64),
}


@pytest.mark.parametrize("name", sorted(LONG))
def test_attention(dev, name):
    a = dict(LONG[name])
    G = a.pop("G")
    c = big_cache(dev, seed=60, **a)
    walks_far(c, G, dev)
    q = C.queries(c, G, 61)
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert out.isfinite().all() and lse.isfinite().all()
    # The longest, ones whose end falls on and beside a slice's, and the last.
    C.check_attention(*part(c, G, q, out, lse, [2, 4, 7, c["B"] // 2, c["B"] - 1], [0, c["Hkv"] - 1]))
    again, lse2, _ = C.attention(c, q)
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # the same bits whichever CTA merges


def rescales(c, G, q, b, h):
    """How often the running maximum of some row of (sequence b, KV head h) has to move while its chunks of 128 keys
    pass in order: by more than 2^8, from the first chunk's on."""
    pools, table, ctx, *_ = C.arrays(c)
    n = int(ctx[b]) // 128 * 128
    K = O.values(O.slots(pools[0], table[b], 0, n)[:, h], O.slots(pools[1], table[b], 0, n)[:, h])
    s = K @ C.np64(q[int(c["cu"][b]), h * G]).astype(np.float64) / np.sqrt(c["D"]) / np.log(2)
    tops = s.reshape(-1, 128).max(1)
    m, moves = tops[0], 0
    for t in tops[1:]:
        if t > m + 8:
            m, moves = t, moves + 1
    return moves


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,k", [(4, 0), (4, 8)])
@pytest.mark.parametrize("rising", [True, False])
def test_attention_moving_scores(dev, rising, G, k, D):
    """Keys that grow along the context move the maxima, and with them the sums and outputs so far, within a CTA's run of
    chunks; keys that shrink leave nearly everything far below the maximum of the first."""
    B = 20
    c = big_cache(dev, [6000] * B, [k] * B, 8, D, 64, 62)
    walks_far(c, G, dev)
    n = c["max_pages"] * 64
    size = torch.linspace(0.05, 40, n) if rising else 30.0 * 0.999 ** torch.arange(n, dtype=torch.float64)
    by = torch.ones((c["pools"][1].shape[0], 64))
    by[c["table"].cpu().long().reshape(-1)] = size.float().reshape(-1, 64).repeat(B, 1)
    c["pools"][1][..., 0] *= by[:, None, :, None].to(dev)
    q = C.queries(c, G, 63)
    if rising:
        sub, q1, *_ = part(c, G, q, q, q[..., 0], [3], [2])
        assert rescales(sub, G, q1, 0, 0) >= 5
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert out.isfinite().all() and lse.isfinite().all()
    C.check_attention(*part(c, G, q, out, lse, [0, 3, B - 1], [0, 2, 7]))


# ---- prompts into the cache, long read-backs ---------------------------------------------------------
PROMPTS = {
    "straddling": dict(ctx=[0, 17, 70], k=[799, 450, 0], Hkv=3, G=5, D=128),             # 21 heads, eight to a warp
    "straddling_d64": dict(ctx=[0, 63, 70], k=[1499, 300, 64], Hkv=5, G=3, D=64, page=128),  # 25 heads, sixteen to a warp
    "few_heads": dict(ctx=[100, 0], k=[4999, 1900], Hkv=1, G=1, D=128),                  # queries, keys and values in one warp
    "few_heads_d64": dict(ctx=[100, 0], k=[5999, 3999], Hkv=1, G=2, D=64),
}


@pytest.mark.parametrize("norms", [(True, True), (False, False), (True, False)])
@pytest.mark.parametrize("name", sorted(PROMPTS))
def test_heads_of_prompts(dev, name, norms):
    a = PROMPTS[name]
    c, x, w, rope, q, st, before, call = _norm_rope(dev, norms=norms, seed=70, **a)
    heads, slots = (a["G"] + 2) * a["Hkv"], 256 // a["D"]
    assert c["R"] * heads // (4 * slots) >= 16 * sms(dev)  # four groups of heads to a warp
    call()
    assert int(st.item()) == 0
    _check_heads(c, x, w, rope, q, before, 1e-6)


def test_prompt_rows_are_the_single_rows(dev):
    """The form for many rows writes the bits that the form for few rows writes."""
    for D, Hkv, G in ((128, 3, 5), (64, 5, 3)):
        a = dict(ctx=[0], k=[1999], Hkv=Hkv, G=G, D=D)
        c, x, w, rope, q, st, before, call = _norm_rope(dev, seed=71, **a)
        call()
        pools, q_many = [t.clone() for t in c["pools"]], q.clone()
        for p, b in zip(c["pools"], before):
            p.copy_(b)
        x = x.reshape(c["R"], -1).to(dev)
        for r in range(0, c["R"], 50):
            few = torch.empty_like(q[r:r + 50])
            ctx = torch.tensor([r], dtype=torch.int32, device=dev)
            kd, cu = torch.tensor([49], dtype=torch.int32, device=dev), torch.tensor([0, 50], dtype=torch.int32, device=dev)
            spade.spade_verify_qk_norm_rope_kv4(x[r:r + 50].contiguous(), *[t.to(dev) for t in w], rope, few, *c["pools"],
                                                c["table"], ctx, kd, cu, eps=1e-6, max_k=49, status=st)
            assert torch.equal(few, q_many[r:r + 50])
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        for a1, b1 in zip(pools, c["pools"]):
            assert torch.equal(a1.view(torch.uint8), b1.view(torch.uint8))


@pytest.mark.parametrize("D,Hkv,page", [(128, 3, 64), (128, 5, 128), (128, 10, 64), (64, 9, 192)])
def test_long_reads(dev, D, Hkv, page):
    """More rows than the grid takes at once, for one to five parts of heads."""
    n = [9000, 1, 5000]
    parts = (Hkv * (D // 8) + 31) // 32
    covered = ((16 * sms(dev) + 2) // 3) * 8 // parts + 1 + 8
    assert n[0] > covered
    c = big_cache(dev, [9100, 100, 5200], [0, 0, 0], Hkv, D, page, 72)
    starts = torch.tensor([99, 70, 1], dtype=torch.int32)
    cu = torch.tensor([0, 9000, 9001, 14001], dtype=torch.int32)
    k = torch.full((14003, Hkv, D), 7.0, dtype=torch.bfloat16, device=dev)
    v, st = k.clone(), spade.status_tensor(dev)
    spade.spade_kv_read_kv4(*c["pools"], c["table"], starts.to(dev), cu.to(dev), k, v, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    pools, table, *_ = C.arrays(c)
    for b in range(3):
        slot = np.arange(int(starts[b]), int(starts[b]) + n[b])
        page_of, at = table[b][slot // page], slot % page
        for i, got in ((0, k), (2, v)):
            want = torch.from_numpy(O.values(pools[i][page_of, :, at], pools[i + 1][page_of, :, at])).to(torch.bfloat16)
            assert torch.equal(got[int(cu[b]):int(cu[b + 1])].cpu(), want)
    assert (k[14001:] == 7).all() and (v[14001:] == 7).all()
