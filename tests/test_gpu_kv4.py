"""The paged 4-bit cache on the GPU: heads normed, rotated and stored, the commit, reading back, and the
attention over it, against float64 and under hostile contents of the slots that nothing may see."""
import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4
from tests import int4_cases as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev(gpu_lib):
    return torch.device("cuda:0")


# ---- heads into the cache ------------------------------------------------------------------------
HEADS = {
    "one_token": dict(ctx=[0], k=[0], Hkv=1, G=1, D=64),
    "odd_heads": dict(ctx=[5, 63, 200], k=[2, 1, 0], Hkv=3, G=1, D=128),
    "grouped": dict(ctx=[64, 127, 0], k=[8, 3, 12], Hkv=2, G=5, D=128),
    "small_heads": dict(ctx=[64, 127, 0], k=[8, 3, 12], Hkv=5, G=3, D=64),
    "prompt": dict(ctx=[0, 17], k=[299, 150], Hkv=2, G=2, D=128, page=128),
    "far": dict(ctx=[32000], k=[4], Hkv=1, G=8, D=128, page=64),
}


def _norm_rope(dev, ctx, k, Hkv, G, D, page=64, norms=(True, True), seed=1, eps=1e-6, scale=1.0):
    c = C.cache(ctx, k, Hkv, D, page, seed, dev)
    g = torch.Generator().manual_seed(seed + 50)
    x = (torch.randn((c["R"], (G + 2) * Hkv, D), generator=g) * scale).to(torch.bfloat16)
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(torch.bfloat16) if on else None for on in norms]
    rope = int4.rope_table(10000.0, D, c["max_pages"] * page, device=dev)
    q = torch.full((c["R"], G * Hkv, D), float("nan"), dtype=torch.bfloat16, device=dev)
    st = spade.status_tensor(dev)
    before = [t.clone() for t in c["pools"]]

    def call(**over):
        a = dict(ctx=c["ctx"], k=c["k"], cu=c["cu"], table=c["table"], rope=rope, max_k=c["max_k"], **over)
        spade.spade_verify_qk_norm_rope_kv4(
            x.reshape(c["R"], -1).to(dev), *[None if t is None else t.to(dev) for t in w], a["rope"], q, *c["pools"],
            a["table"], a["ctx"], a["k"], a["cu"], eps=eps, max_k=a["max_k"], status=st)
        torch.cuda.synchronize()

    return c, x, w, rope, q, st, before, call


def _written(c):
    """Which (page, slot) the blocks of the sequences cover."""
    m = torch.zeros(c["pools"][0].shape[:1] + (c["page"],), dtype=torch.bool)
    table = c["table"].cpu()
    for b in range(c["B"]):
        for s in range(int(c["ctx"][b]), int(c["ctx"][b] + c["k"][b]) + 1):
            m[int(table[b, s // c["page"]]), s % c["page"]] = True
    return m


def _check_heads(c, x, w, rope, q, before, eps, seqs=None):
    Hkv, D = c["Hkv"], c["D"]
    Hq = x.shape[1] - 2 * Hkv
    pools, table, ctx, k, cu = C.arrays(c)
    t = C.np64(rope)
    for b in range(c["B"]) if seqs is None else seqs:
        rows = slice(int(cu[b]), int(cu[b + 1]))
        turn = t[int(ctx[b]):int(ctx[b] + k[b]) + 1]
        xs = C.np64(x[rows])
        ws = [None if v is None else C.np64(v) for v in w]
        want, size = O.turned(xs[:, :Hq], ws[0], turn, eps)
        # bf16 rounds once; before it the norm (a sum of D, a root, two products) and the rotation lose a few ulps.
        fp32 = 2.0 ** -20 * size + 1e-37
        assert (np.abs(C.np64(q[rows]) - want) <= 2.0 ** -8 * np.abs(want) + fp32).all()
        want, size = O.turned(xs[:, Hq:Hq + Hkv], ws[1], turn, eps)
        got = [O.slots(pool, table[b], int(ctx[b]), int(k[b]) + 1) for pool in pools]
        assert O.check_quantised(want, 2.0 ** -20 * size + 1e-37, got[0], got[1].astype(np.float32)) == 0
        codes, params = int4.quantize(x[rows, Hq + Hkv:].float(), 64)  # values as they are: the same operations
        assert np.array_equal(got[2], codes.numpy()) and np.array_equal(got[3], params.numpy(), equal_nan=True)
    # Every other slot is as it was.
    rest = ~_written(c)[:, None].expand(-1, Hkv, -1)
    for a, p in zip(before, c["pools"]):
        assert torch.equal(a.cpu().view(torch.uint8)[rest], p.cpu().view(torch.uint8)[rest])


@pytest.mark.parametrize("norms", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("name", sorted(HEADS))
def test_heads(dev, name, norms):
    c, x, w, rope, q, st, before, call = _norm_rope(dev, norms=norms, **HEADS[name])
    call()
    assert int(st.item()) == 0
    _check_heads(c, x, w, rope, q, before, 1e-6)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 1e4])
def test_heads_of_any_size(dev, scale):
    """Values whose scales leave float16's normal range on either side; a large eps."""
    c, x, w, rope, q, st, before, call = _norm_rope(dev, scale=scale, eps=0.5, **HEADS["grouped"])
    call()
    assert int(st.item()) == 0
    _check_heads(c, x, w, rope, q, before, 0.5)


def test_heads_not_finite(dev):
    """A NaN or an infinity poisons its own group of the key or value, its query head, and nothing else."""
    c, x, w, rope, q, st, before, call = _norm_rope(dev, norms=(False, False), **HEADS["odd_heads"])
    x[0, 1, 3], x[1, 3, 70], x[2, 8, 5] = float("nan"), float("inf"), -float("inf")  # a query, a key, a value head
    call()
    bad = q.cpu().isnan().any(-1)
    assert bad.nonzero().tolist() == [[0, 1]]
    pools, table, ctx, k, cu = C.arrays(c)
    kp, vp = (O.slots(p, table[0], int(ctx[0]), 3) for p in (pools[1], pools[3]))
    # (a key pair (j, j + 64) shares the infinity: both of its groups are poisoned)
    assert np.argwhere(np.isnan(kp[..., 0])).tolist() == [[1, 0, 0], [1, 0, 1]]
    assert np.argwhere(np.isnan(vp[..., 0])).tolist() == [[2, 2, 0]]


@pytest.mark.parametrize("fault", ["ctx", "draft", "rows", "capacity", "table_end", "page"])
def test_heads_reported(dev, fault):
    """A sequence that cannot be stored is skipped and named; the others are stored."""
    c, x, w, rope, q, st, before, call = _norm_rope(dev, ctx=[5, 63, 100], k=[2, 1, 0], Hkv=2, G=2, D=128)
    keep = {n: c[n].clone() for n in ("ctx", "k", "cu", "table")}
    want = spade.DEV_BAD_INDEX
    if fault == "ctx":
        c["ctx"][1] = -1
    elif fault == "draft":
        c["k"][1] = c["max_k"] + 1
    elif fault == "rows":
        c["cu"][2] += 1
    elif fault == "capacity":
        c["ctx"][1] = c["max_pages"] * 64 - 1
        want = spade.DEV_CAPACITY
    elif fault == "page":
        c["table"][1, 0] = c["pools"][0].shape[0]
        c["table"][1, 1] = -1
    rope_given = rope[:64].contiguous() if fault == "table_end" else rope
    spade.spade_verify_qk_norm_rope_kv4(x.reshape(c["R"], -1).to(dev), *[t.to(dev) for t in w], rope_given, q, *c["pools"],
                                        c["table"], c["ctx"], c["k"], c["cu"], eps=1e-6, max_k=c["max_k"], status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == want
    good = {"rows": [0], "table_end": [0]}.get(fault, [0, 2])
    c.update(keep)
    written = _written(c)
    for b in set(range(3)) - set(good):  # (nothing of theirs is written)
        for s in range(int(keep["ctx"][b]), int(keep["ctx"][b] + keep["k"][b]) + 1):
            written[int(keep["table"][b, s // 64]), s % 64] = False
        if fault != "page":
            assert q[int(keep["cu"][b]):int(keep["cu"][b + 1])].isnan().all()
    rest = ~written[:, None].expand(-1, 2, -1)
    for a, p in zip(before, c["pools"]):
        assert torch.equal(a.cpu().view(torch.uint8)[rest], p.cpu().view(torch.uint8)[rest])
    pools, table, ctx, k, cu = C.arrays(c)
    for b in good:
        rows = slice(int(cu[b]), int(cu[b + 1]))
        codes, params = int4.quantize(x[rows, 6:].float(), 64)
        got = [O.slots(p, table[b], int(ctx[b]), int(k[b]) + 1) for p in pools[2:]]
        assert np.array_equal(got[0], codes.numpy()) and np.array_equal(got[1], params.numpy())


# ---- commit and read -----------------------------------------------------------------------------
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_commit(dev, D, in_place):
    c = C.cache([0, 60, 127, 64, 300], [0, 8, 3, 5, 16], 3, D, 64, 11, dev)
    acc = torch.tensor([0, 2, 3, 0, 7], dtype=torch.int32, device=dev)
    before = [t.clone() for t in c["pools"]]
    ctx0 = c["ctx"].clone()
    new = c["ctx"] if in_place else torch.full_like(c["ctx"], -9)
    st = spade.status_tensor(dev)
    spade.spade_kv_commit_kv4(*c["pools"], c["table"], c["ctx"], acc, c["k"], new, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(new, ctx0 + acc + 1)
    if not in_place:
        assert torch.equal(c["ctx"], ctx0)
    cleared = torch.zeros(before[0].shape[0], 64, dtype=torch.bool)
    table = c["table"].cpu()
    for b in range(5):
        for s in range(int(ctx0[b] + acc[b]) + 1, int(ctx0[b] + c["k"][b]) + 1):
            cleared[int(table[b, s // 64]), s % 64] = True
    m = cleared[:, None].expand(-1, 3, -1)
    for a, p in zip(before, c["pools"]):
        a, p = a.cpu().view(torch.uint8), p.cpu().view(torch.uint8)
        assert torch.equal(a[~m], p[~m]) and not p[m].any()


@pytest.mark.parametrize("fault", ["accepted", "draft", "capacity", "page"])
def test_commit_reported(dev, fault):
    c = C.cache([60, 10, 70], [8, 3, 2], 2, 128, 64, 12, dev)
    acc = torch.tensor([2, 1, 0], dtype=torch.int32, device=dev)
    table, ctx, k = c["table"].clone(), c["ctx"].clone(), c["k"].clone()
    if fault == "accepted":
        acc[0] = 9
    elif fault == "draft":
        k[0] = -1
    elif fault == "capacity":
        ctx[0] = c["max_pages"] * 64 - 8
    else:
        table[0, 1] = -1
    before = [t.clone() for t in c["pools"]]
    new, st = torch.full_like(ctx, -9), spade.status_tensor(dev)
    spade.spade_kv_commit_kv4(*c["pools"], table, ctx, acc, k, new, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == (spade.DEV_CAPACITY if fault == "capacity" else spade.DEV_BAD_INDEX)
    assert new.tolist() == [int(ctx[0]), 12, 71]
    pages = c["table"][0].long().cpu()  # the reported sequence's own pages
    for a, p in zip(before, c["pools"]):
        assert torch.equal(a.cpu()[pages].view(torch.uint8), p.cpu()[pages].view(torch.uint8))


@pytest.mark.parametrize("D,Hkv,page", [(64, 1, 64), (128, 3, 64), (128, 8, 256)])
def test_read(dev, D, Hkv, page):
    c = C.cache([0, 100, 700], [3, 60, 0], Hkv, D, page, 13, dev, poison=False)
    starts = torch.tensor([1, 0, 650], dtype=torch.int32)
    n = [3, 161, 0]
    cu = torch.tensor([0, 3, 164, 164], dtype=torch.int32)
    k = torch.full((170, Hkv, D), 7.0, dtype=torch.bfloat16, device=dev)
    v, st = k.clone(), spade.status_tensor(dev)
    spade.spade_kv_read_kv4(*c["pools"], c["table"], starts.to(dev), cu.to(dev), k, v, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    pools, table, *_ = C.arrays(c)
    for b in range(3):
        for i, out in ((0, k), (2, v)):
            if n[b]:
                want = O.values(O.slots(pools[i], table[b], int(starts[b]), n[b]),
                                O.slots(pools[i + 1], table[b], int(starts[b]), n[b]))
                got = out[int(cu[b]):int(cu[b + 1])].cpu()
                assert torch.equal(got, torch.from_numpy(want).to(torch.bfloat16))
    assert (k[164:] == 7).all() and (v[164:] == 7).all()


def test_read_reported(dev):
    c = C.cache([10, 10, 10, 10], [3, 3, 3, 3], 2, 128, 64, 14, dev, poison=False)
    starts = torch.tensor([-1, 62, 0, 0], dtype=torch.int32, device=dev)  # before the start, past the end
    cu = torch.tensor([0, 4, 8, 12, 16], dtype=torch.int32, device=dev)
    c["table"][2, 0] = 99  # not in the pool: zeros
    k = torch.full((16, 2, 128), 7.0, dtype=torch.bfloat16, device=dev)
    v, st = k.clone(), spade.status_tensor(dev)
    spade.spade_kv_read_kv4(*c["pools"], c["table"], starts, cu, k, v, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == spade.DEV_BAD_INDEX | spade.DEV_CAPACITY
    for out in (k, v):
        assert (out[:8] == 7).all() and (out[8:12] == 0).all() and (out[12:] != 7).any()


# ---- attention -------------------------------------------------------------------------------------
ATTENTION = {
    "one_key": dict(ctx=[0], k=[0], Hkv=1, G=1, D=64),
    "one_token_each": dict(ctx=[0, 1, 63, 64, 127, 128, 500], k=[0] * 7, Hkv=2, G=4, D=128),
    "edges": dict(ctx=[62, 63, 64, 126, 127, 128], k=[1, 2, 0, 3, 5, 1], Hkv=2, G=2, D=128),
    "edges_d64": dict(ctx=[62, 63, 64, 126, 127, 128], k=[1, 2, 0, 3, 5, 1], Hkv=2, G=2, D=64),
    "no_context": dict(ctx=[0, 0, 0], k=[0, 4, 12], Hkv=1, G=3, D=128),
    "rows_17": dict(ctx=[300], k=[16], Hkv=2, G=1, D=128),
    "rows_33": dict(ctx=[300], k=[10], Hkv=1, G=3, D=64),
    "rows_55": dict(ctx=[700, 3], k=[10, 0], Hkv=3, G=5, D=128),
    "rows_64": dict(ctx=[190], k=[7], Hkv=2, G=8, D=128),
    "two_row_blocks": dict(ctx=[200, 50], k=[12, 3], Hkv=2, G=8, D=128),
    "block_in_blocks": dict(ctx=[10], k=[149], Hkv=1, G=2, D=64),
    "large_pages": dict(ctx=[1000, 257, 5], k=[4, 0, 8], Hkv=2, G=5, D=128, page=256),
    "odd_pages": dict(ctx=[400, 191], k=[4, 0], Hkv=2, G=7, D=128, page=192),
    "split_keys": dict(ctx=[9000], k=[3], Hkv=1, G=8, D=128),
    "split_keys_d64": dict(ctx=[9000], k=[3], Hkv=1, G=4, D=64),
    "many": dict(ctx=list(range(0, 600, 15)), k=[i % 4 for i in range(40)], Hkv=1, G=2, D=128),
}


@pytest.mark.parametrize("name", sorted(ATTENTION))
def test_attention(dev, name):
    a = dict(ATTENTION[name])
    G = a.pop("G")
    c = C.cache(page=a.pop("page", 64), seed=20, dev=dev, **a)
    q = C.queries(c, G, 21)
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    C.check_attention(c, q, out, lse)


@pytest.mark.parametrize("sharp,scale", [(30.0, 1.0), (1e-3, 1.0), (1.0, 1e-5), (1.0, 300.0), (1e30, 1e-3), (300.0, 20.0)])
def test_attention_of_any_size(dev, sharp, scale):
    """One key that takes all, flat rows, values and scores far from 1."""
    c = C.cache([500, 70], [3, 2], 2, 128, 64, 22, dev, scale=scale)
    q = C.queries(c, 4, 23, sharp=sharp)
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    C.check_attention(c, q, out, lse)


def test_attention_rising_scores(dev):
    """Row maxima that move at every tile: keys that grow along the context."""
    c = C.cache([1500], [3], 1, 128, 64, 24, dev)
    n = 1504
    rise = torch.linspace(0, 40, n)
    kp = c["pools"][1].cpu()
    for s in range(n):
        kp[int(c["table"][0, s // 64]), 0, s % 64, :, 0] *= rise[s]
    c["pools"][1].copy_(kp)
    q = C.queries(c, 4, 25)
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    C.check_attention(c, q, out, lse)


def test_attention_falling_scores(dev):
    """The largest scores come first: what follows is far below the maximum."""
    c = C.cache([1500], [3], 1, 128, 64, 26, dev)
    kp = c["pools"][1].cpu()
    for s in range(1504):
        kp[int(c["table"][0, s // 64]), 0, s % 64, :, 0] *= 30.0 * (0.99 ** s)
    c["pools"][1].copy_(kp)
    q = C.queries(c, 4, 27)
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    C.check_attention(c, q, out, lse)


@pytest.mark.parametrize("which", [1, 3])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_attention_poisoned_draft(dev, which, value):
    """A draft whose key or value is not finite reaches the rows that see it, and no other row or head."""
    c = C.cache([100, 40], [5, 2], 2, 128, 64, 28, dev)
    q = C.queries(c, 3, 29)
    clean, _, _ = C.attention(c, q)
    torch.cuda.synchronize()
    s = 103  # draft position 3 of sequence 0, KV head 1
    c["pools"][which][int(c["table"][0, s // 64]), 1, s % 64, 1, 0] = value
    out, lse, st = C.attention(c, q)
    torch.cuda.synchronize()
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    bad[3:6, 3:] = True
    assert torch.equal(out.cpu().isnan().any(-1), bad)
    assert torch.equal(out.cpu()[~bad], clean.cpu()[~bad])
    assert torch.equal(lse.cpu().isnan(), bad)


def test_attention_query_not_finite(dev):
    """A query row with a NaN is NaN; the others are as they were."""
    c = C.cache([100, 40], [5, 2], 2, 128, 64, 30, dev)
    q = C.queries(c, 3, 31)
    clean, _, _ = C.attention(c, q)
    q2 = q.clone()
    q2[4, 2, 77] = float("nan")
    out, _, _ = C.attention(c, q2)
    torch.cuda.synchronize()
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    bad[4, 2] = True
    assert out.cpu()[bad].isnan().all() and torch.equal(out.cpu()[~bad], clean.cpu()[~bad])


@pytest.mark.parametrize("fault", ["ctx", "draft", "rows", "capacity"])
def test_attention_reported(dev, fault):
    c = C.cache([100, 40, 64], [5, 2, 3], 2, 128, 64, 32, dev)
    q = C.queries(c, 3, 33)
    rows, good = list(range(6, 9)), [0, 2]
    if fault == "ctx":
        c["ctx"][1] = -5
    elif fault == "draft":
        c["k"][1] = 6
    elif fault == "rows":
        c["cu"][3] += 5
        rows, good = list(range(9, 13)), [0, 1]
    else:
        c["ctx"][1] = 127
    out, _, st = C.attention(c, q, max_k=5)
    torch.cuda.synchronize()
    assert int(st.item()) == (spade.DEV_CAPACITY if fault == "capacity" else spade.DEV_BAD_INDEX)
    assert out[rows].isnan().all()
    # The others (their keys may be split over the GPU in another way than without the fault) against float64.
    at = [r for b in good for r in range(int(c["cu"][b]), int(c["cu"][b]) + int(c["k"][b]) + 1)]
    rest = dict(c, table=c["table"][good], ctx=c["ctx"][good], k=c["k"][good], B=2)
    rest["cu"] = C.lengths(rest["ctx"].tolist(), rest["k"].tolist())[2]
    C.check_attention(rest, q[at], out[at], None)


def test_attention_bad_page_reads_zeros(dev):
    """A table entry outside the pool is reported and read as zeros."""
    c = C.cache([100], [2], 2, 128, 64, 34, dev)
    q = C.queries(c, 3, 35)
    zeroed = dict(c, pools=[t.clone() for t in c["pools"]])
    page = int(c["table"][0, 0])
    for t in zeroed["pools"]:
        t[page] = 0
    want, wlse, _ = C.attention(zeroed, q)
    for bad in (-1, c["pools"][0].shape[0], 1 << 30):
        c["table"][0, 0] = bad
        out, lse, st = C.attention(c, q)
        torch.cuda.synchronize()
        assert int(st.item()) == spade.DEV_BAD_INDEX
        assert torch.equal(out, want) and torch.equal(lse, wlse)


def test_attention_calls_share_a_workspace(dev):
    """Calls of different sizes, one after the other on one workspace and on another stream: the same bits."""
    cases = [C.cache([3000, 40], [3, 1], 2, 128, 64, 36, dev), C.cache([70] * 9, [0] * 9, 1, 64, 64, 37, dev)]
    qs = [C.queries(c, 4, 38 + i) for i, c in enumerate(cases)]
    first = [C.attention(c, q)[0].clone() for c, q in zip(cases, qs)]
    size = max(spade.spade_attn_workspace_size(c["B"], 4 * c["Hkv"], c["Hkv"], c["D"], c["max_pages"] * 64, c["max_k"])
               for c in cases)
    ws = torch.zeros(size, dtype=torch.uint8, device=dev)
    stream = torch.cuda.Stream(dev)
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for c, q, f in zip(cases, qs, first):
            with torch.cuda.stream(stream):
                out, _, st = C.attention(c, q, workspace=ws)
            stream.synchronize()
            assert torch.equal(out, f) and int(st.item()) == 0


def test_attention_without_lse_and_loose_bound(dev):
    """No lse asked for; a max_k above every block: the same output."""
    c = C.cache([130, 7], [2, 4], 2, 128, 64, 40, dev)
    q = C.queries(c, 2, 41)
    out, _, _ = C.attention(c, q)
    alone, none, st = C.attention(c, q, max_k=40, lse=False)
    torch.cuda.synchronize()
    assert none is None and int(st.item()) == 0
    C.check_attention(c, q, alone, None)
    C.check_attention(c, q, out, None)


def test_attention_workspace_refused(dev):
    c = C.cache([130], [2], 2, 128, 64, 42, dev)
    q = C.queries(c, 2, 43)
    with pytest.raises(spade.SpadeError) as e:
        C.attention(c, q, workspace=torch.zeros(256, dtype=torch.uint8, device=dev))
    assert e.value.status == 6


def test_attention_in_a_graph(dev):
    """Captured and replayed with new contents: what a plain call gives."""
    c = C.cache([3000, 40], [3, 1], 2, 128, 64, 44, dev)
    q, q2 = C.queries(c, 4, 45), C.queries(c, 4, 46)
    want = C.attention(c, q2)[0].clone()
    ws = spade.attn_workspace(c["B"], 8, 2, 128, c["max_pages"] * 64, c["max_k"], device=dev)
    out, st = torch.empty_like(q), spade.status_tensor(dev)
    stream = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        spade.spade_verify_attention_kv4(q, *c["pools"], c["table"], c["ctx"], c["k"], c["cu"], out, None,
                                         max_k=c["max_k"], workspace=ws, status=st)
    q.copy_(q2)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and int(st.item()) == 0
