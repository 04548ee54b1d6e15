"""The tree verify step's calls at the ends of what they take: offsets past 32 bits, the most sequences, rows and nodes,
padded batches, shared pages, calls beside one another, a whole step in a graph."""
import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from tests import tree_cases as T
from tests.test_gpu_sample import check as check_sample

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _block(c, G, seed, freq):
    """One block through the rotary write, the attention and the commit: every output, and the block's slots."""
    gen = torch.Generator().manual_seed(seed)
    k, Hkv, D = c["n"].cpu(), c["Hkv"], c["D"]
    par = T.parents(k, "tree", seed)
    mask = T.tree_mask(par, k, c["cu"].cpu()).to(DEV)
    x = torch.randn((c["R"], (G + 2) * Hkv * D), generator=gen).to(torch.bfloat16).to(DEV)
    q = torch.empty((c["R"], G * Hkv, D), dtype=torch.bfloat16, device=DEV)
    st = spade.status_tensor(DEV)
    lens = (c["ctx"], c["n"], c["cu"])
    tokens = torch.randint(0, 3, (c["R"],), generator=gen, dtype=torch.int32).to(DEV)
    drafts = torch.randint(0, 3, (c["R"] - c["B"],), generator=gen, dtype=torch.int32).to(DEV)
    acc, nxt, new = (torch.empty(c["B"], dtype=torch.int32, device=DEV) for _ in range(3))
    path = torch.empty(c["R"], dtype=torch.int32, device=DEV)
    if c["page"]:
        spade.spade_verify_rope_paged(x, freq, None, c["table"], *lens, q, c["k"], c["v"], max_k=c["max_k"], status=st)
    else:
        spade.spade_verify_rope(x, freq, None, *lens, q, c["k"], c["v"], max_k=c["max_k"], status=st)
    out, lse, st2 = T.attention(c, q, mask)
    block = (c["ctx"], par.to(DEV), drafts, tokens, c["n"], c["cu"], acc, nxt, path, new)
    if c["page"]:
        spade.spade_tree_commit_paged(c["k"], c["v"], c["table"], *block, max_k=c["max_k"], status=st)
    else:
        spade.spade_tree_commit(c["k"], c["v"], *block, max_k=c["max_k"], status=st)
    assert int(st.item()) == 0 and int(st2.item()) == 0
    slots = []
    for b in range(c["B"]):
        at = torch.arange(int(c["ctx"][b]) + int(k[b]) + 1, device=DEV)
        for m in ("k", "v"):
            slots.append(c[m][c["table"][b].long()[at // c["page"]], :, at % c["page"]] if c["page"] else c[m][b][:, at])
    return [q, out, lse, acc, nxt, path, new] + slots


def test_pages_far_into_a_pool(gpu_lib):
    """Rows of the cache whose offsets in elements pass 2^32: what a small pool gives, bit by bit."""
    near = T.cache([300, 70], [40, 9], 1, 128, 64, 1, DEV)
    num = 640_000  # pages: 41 million rows of 128
    shift = num - near["k"].shape[0]
    far = dict(near, table=near["table"] + shift)
    for m in ("k", "v"):
        far[m] = torch.empty((num, 1, 64, 128), dtype=torch.bfloat16, device=DEV)
        far[m][shift:].copy_(near[m])
    assert (shift * 64) * 128 > 2 ** 32
    freq = spade.rope.inv_freq(10000.0, 128)
    a = _block(near, 4, 2, freq)
    for x, y in zip(a, _block(far, 4, 2, freq)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_a_long_dense_cache(gpu_lib):
    near = T.cache([30, 10, 200], [3, 0, 40], 1, 128, 0, 3, DEV)
    far = dict(near, cap=2 ** 24 + 8)
    for m in ("k", "v"):
        far[m] = torch.empty((3, 1, far["cap"], 128), dtype=torch.bfloat16, device=DEV)
        far[m][:, :, :near["cap"]].copy_(near[m])
    assert 2 * far["cap"] * 128 > 2 ** 32
    freq = spade.rope.inv_freq(10000.0, 64)
    a = _block(near, 2, 4, freq)
    for x, y in zip(a, _block(far, 2, 4, freq)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_rows_far_apart(gpu_lib):
    """Logits and projections whose rows lie gigabytes apart."""
    big = torch.empty(5 * 2 ** 30, dtype=torch.float16, device=DEV)
    x = big.as_strided((5, 4001), (2 ** 30, 1), 3)
    gen = torch.Generator().manual_seed(5)
    x.copy_(torch.randn((5, 4001), generator=gen) * 3)
    u = np.random.RandomState(6).rand(5).astype(np.float32)
    tok, ch = torch.empty(5, dtype=torch.int32, device=DEV), torch.empty(5, device=DEV)
    st = spade.status_tensor(DEV)
    spade.spade_sample(x, torch.from_numpy(u).to(DEV), tok, None, ch, top_p=torch.full((5,), 0.9, device=DEV), status=st)
    assert int(st.item()) == 0
    check_sample(x, u, tok, None, ch, top_p=0.9, loose=2.0 ** -20 + 2.0 ** -21)

    c = T.cache([9], [4], 1, 64, 0, 7, DEV)
    qkv = big.view(torch.bfloat16).as_strided((5, 4 * 64), (2 ** 30, 1))
    qkv.copy_(torch.randn((5, 4 * 64), generator=gen))
    q = [torch.empty((5, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    freq = spade.rope.inv_freq(10000.0, 64)
    caches = []
    for y, rows in zip(q, (qkv, qkv.contiguous())):
        k, v = c["k"].clone(), c["v"].clone()
        spade.spade_verify_rope(rows, freq, None, c["ctx"], c["n"], c["cu"], y, k, v, max_k=4, status=st)
        caches += [k, v]
    assert torch.equal(q[0], q[1]) and int(st.item()) == 0
    for a, b in zip(caches[:2], caches[2:]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_most_sequences(gpu_lib):
    """The attention's 512 sequences, among them ones without context."""
    rng = np.random.RandomState(8)
    ctx, k = rng.randint(0, 90, 512).tolist(), rng.randint(0, 5, 512).tolist()
    c = T.cache(ctx, k, 1, 64, 64, 9, DEV)
    q = T.queries(c, 2, 10)
    mask = T.tree_mask(T.parents(k, "tree", 11), k, c["cu"].cpu())
    out, lse, st = T.attention(c, q, mask)
    assert int(st.item()) == 0
    T.check_attention(c, q, mask, out, lse)


@pytest.mark.parametrize("V,dtype", [(786_000, torch.float32), (1_500_000, torch.bfloat16)])
@pytest.mark.parametrize("opts", [dict(), dict(top_k=40, top_p=0.9), dict(top_p=0.5), dict(temperature=0.5, min_p=0.2)], ids=str)
def test_longest_rows(gpu_lib, V, dtype, opts):
    gen = torch.Generator(device=DEV).manual_seed(12)
    x = (torch.randn((3, V), generator=gen, device=DEV) * 3).to(dtype)
    u = np.random.RandomState(13).rand(3).astype(np.float32)
    put = {n: torch.full((3,), v, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV) for n, v in opts.items()}
    tok, ch, probs = torch.empty(3, dtype=torch.int32, device=DEV), torch.empty(3, device=DEV), torch.empty((3, V), device=DEV)
    st = spade.status_tensor(DEV)
    spade.spade_sample(x, torch.from_numpy(u).to(DEV), tok, probs, ch, status=st, **put)
    assert int(st.item()) == 0
    check_sample(x, u, tok, probs, ch, **opts)


def test_most_rows(gpu_lib):
    """65535 rows of a few tokens: each its own draw."""
    R = 65535
    x = torch.tensor([0.0, 1.0, 2.0], device=DEV).repeat(R, 1)
    u = (torch.arange(R, device=DEV, dtype=torch.float64) / R).float()
    tok = torch.empty(R, dtype=torch.int32, device=DEV)
    st = spade.status_tensor(DEV)
    spade.spade_sample(x, u, tok, status=st)
    p = torch.softmax(x[0].double(), 0).cumsum(0)
    want = (u.double()[:, None] >= p[None, :]).sum(1)
    # (A uniform within 2^-30 of an edge may go either way; the grid of these has none.)
    assert float((u.double()[:, None] - p[None, :]).abs()[:, :2].min()) > 2.0 ** -30
    assert torch.equal(tok.long(), want) and int(st.item()) == 0


@pytest.mark.parametrize("shape", ["chain", "star"])
def test_largest_trees(gpu_lib, shape):
    """16384 nodes: a chain that is accepted whole, and a star whose last leaf is."""
    n = 16384
    par = torch.arange(-1, n - 1, dtype=torch.int32) if shape == "chain" else torch.zeros(n, dtype=torch.int32)
    par[0] = -1
    ctx, kd = torch.tensor([5], dtype=torch.int32, device=DEV), torch.tensor([n - 1], dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    pos = torch.empty(n, dtype=torch.int32, device=DEV)
    mask = torch.empty((n, 512), dtype=torch.int32, device=DEV)
    st = spade.status_tensor(DEV)
    spade.spade_tree_layout(par.to(DEV), ctx, kd, cu, pos, mask, max_k=n - 1, status=st)
    i = torch.arange(n, device=DEV)
    bits = (mask[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32) & 1).reshape(n, n).bool()
    if shape == "chain":
        assert torch.equal(pos, (5 + i).int()) and torch.equal(bits, i[None, :] <= i[:, None])
        drafts = torch.arange(1, n, dtype=torch.int32)
        tokens = torch.arange(1, n + 1, dtype=torch.int32)
    else:
        assert torch.equal(pos, 5 + (i > 0).int()) and torch.equal(bits, (i[None, :] == i[:, None]) | (i[None, :] == 0))
        drafts = torch.arange(1, n, dtype=torch.int32)
        tokens = torch.full((n,), n - 1, dtype=torch.int32)
    k = torch.randn((1, 1, n + 5, 64), device=DEV).to(torch.bfloat16)
    v, was = k * 2, k.clone()
    acc, nxt, new = (torch.empty(1, dtype=torch.int32, device=DEV) for _ in range(3))
    path = torch.empty(n, dtype=torch.int32, device=DEV)
    spade.spade_tree_commit(k, v, ctx, par.to(DEV), drafts.to(DEV), tokens.to(DEV), kd, cu, acc, nxt, path, new, max_k=n - 1,
                            status=st)
    assert int(st.item()) == 0
    if shape == "chain":
        assert int(acc) == n - 1 and int(nxt) == n and int(new) == n + 5 and torch.equal(path, i.int())
        assert torch.equal(k, was) and torch.equal(v, was * 2)
    else:
        assert int(acc) == 1 and int(nxt) == n - 1 and int(new) == 7 and path[:3].tolist() == [0, n - 1, -1]
        assert torch.equal(k[0, 0, 6], was[0, 0, n + 4]) and torch.equal(v[0, 0, 6], was[0, 0, n + 4] * 2)
        assert torch.equal(k[0, 0, :6], was[0, 0, :6]) and int((k[0, 0, 7:] != 0).sum()) == 0


def test_rows_behind_the_last_sequence_stay(gpu_lib):
    """Batches padded to more rows than their sequences have."""
    ctx, k, pad = [20, 90], [5, 33], 9
    c = T.cache(ctx, k, 2, 128, 64, 14, DEV)
    R, full = c["R"], c["R"] + pad
    par = torch.cat([T.parents(k, "tree", 15), torch.full((pad,), 1234, dtype=torch.int32)]).to(DEV)
    lens = (c["ctx"], c["n"], c["cu"])
    st = spade.status_tensor(DEV)
    pos, mask = torch.full((full,), 77, dtype=torch.int32, device=DEV), torch.full((full, 2), 77, dtype=torch.int32, device=DEV)
    spade.spade_tree_layout(par, *lens, pos, mask, max_k=33, status=st)
    gen = torch.Generator().manual_seed(16)
    x = torch.randn((full, 8 * 128), generator=gen).to(torch.bfloat16).to(DEV)
    q, out = (torch.full((full, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse = torch.full((full, 4), 7.0, device=DEV)
    before = {m: c[m].clone() for m in ("k", "v")}
    spade.spade_verify_rope_paged(x, spade.rope.inv_freq(1e4, 128), pos, c["table"], *lens, q, c["k"], c["v"], max_k=33, status=st)
    for m in ("k", "v"):  # as many rows as live nodes were written, no more
        assert int((c[m].view(torch.int16) != before[m].view(torch.int16)).any(-1).any(1).sum()) == R
    spade.spade_verify_attention_tree_paged(q, c["k"], c["v"], c["table"], *lens, mask, out, lse, max_k=33, status=st,
                                            workspace=spade.tree_attn_workspace(2, 4, 2, 128, c["cap"], 33))
    path = torch.full((full,), 77, dtype=torch.int32, device=DEV)
    acc, nxt, new = (torch.empty(2, dtype=torch.int32, device=DEV) for _ in range(3))
    zeros = torch.zeros(full, dtype=torch.int32, device=DEV)
    spade.spade_tree_commit_paged(c["k"], c["v"], c["table"], c["ctx"], par, zeros[:full - 2], zeros, c["n"], c["cu"], acc, nxt,
                                  path, new, max_k=33, status=st)
    assert int(st.item()) == 0
    for t, value in ((pos, 77), (mask, 77), (q, 7.0), (out, 7.0), (lse, 7.0), (path, 77)):
        assert bool((t[R:] == value).all()) and not bool((t[:R] == value).all())


def test_sequences_that_share_their_context(gpu_lib):
    """Two sequences on the same pages of context, each with its own last page for its block."""
    k = [30, 11]
    c = T.cache([128, 128], k, 2, 128, 64, 17, DEV)
    own = c["table"].clone()
    c["table"][1, :2] = c["table"][0, :2]
    q = T.queries(c, 4, 18)
    mask = T.tree_mask(T.parents(k, "tree", 19), k, c["cu"].cpu())
    out, lse, st = T.attention(c, q, mask)
    for m in ("k", "v"):
        c[m][own[1, :2].long()] = c[m][own[0, :2].long()]
    c["table"] = own
    want, wl, _ = T.attention(c, q, mask)
    assert torch.equal(out, want) and torch.equal(lse, wl) and int(st.item()) == 0


def _step(s, stream=None):
    """One verify step of two layers on the state's buffers."""
    lens = (s["ctx"], s["n"], s["cu"])
    more = dict(max_k=s["max_k"], status=s["st"], stream=stream)
    spade.spade_tree_layout(s["par"], *lens, s["pos"], s["mask"], **more)
    for i in range(2):
        kv = s["k"][i], s["v"][i]
        spade.spade_verify_rope_paged(s["x"][i], s["freq"], s["pos"], s["table"], *lens, s["q"], *kv, **more)
        spade.spade_verify_attention_tree_paged(s["q"], *kv, s["table"], *lens, s["mask"], s["out"][i], s["lse"][i],
                                                workspace=s["ws"], **more)
    spade.spade_sample(s["logits"], s["u"], s["tokens"], None, s["chosen"], top_p=s["top_p"], status=s["st"], stream=stream)
    spade.spade_tree_commit_paged(s["k"], s["v"], s["table"], s["ctx"], s["par"], s["drafts"], s["tokens"], s["n"], s["cu"],
                                  s["acc"], s["next"], s["path"], s["ctx"], **more)


def _state(seed):
    ctx, k = [40, 0, 700], [20, 7, 40]
    c = T.cache(ctx, k, 2, 128, 64, 20, DEV, layers=2)
    R = c["R"]
    gen = torch.Generator().manual_seed(seed)
    empty = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device=DEV)
    s = dict(c, par=T.parents(k, "tree", 21).to(DEV), pos=empty(R), mask=empty(R, 2), st=spade.status_tensor(DEV),
             freq=spade.rope.inv_freq(1e4, 128), x=torch.randn((2, R, 10 * 128), generator=gen).to(torch.bfloat16).to(DEV),
             q=empty(R, 6, 128, dtype=torch.bfloat16), out=empty(2, R, 6, 128, dtype=torch.bfloat16),
             lse=empty(2, R, 6, dtype=torch.float32), tokens=empty(R), chosen=empty(R, dtype=torch.float32), acc=empty(3),
             next=empty(3), path=empty(R), ws=spade.tree_attn_workspace(3, 6, 2, 128, c["cap"], 40),
             logits=torch.randn((R, 5003), generator=gen).to(torch.bfloat16).to(DEV), u=torch.rand(R, generator=gen).to(DEV),
             top_p=torch.full((R,), 0.9, device=DEV), drafts=torch.randint(0, 5003, (R - 3,), generator=gen, dtype=torch.int32).to(DEV))
    s["logits"][:, 17] = 12.0  # a likely token, which some drafts have
    s["drafts"][::2] = 17
    return s


RESULTS = ("pos", "mask", "q", "out", "lse", "tokens", "chosen", "acc", "next", "path", "ctx", "k", "v")


def _same(a, b):
    for m in RESULTS:
        assert torch.equal(a[m].view(torch.uint8), b[m].view(torch.uint8)), m


def test_a_step_in_a_graph(gpu_lib):
    """A captured step, replayed on inputs of its own: what the calls give one by one."""
    a, b, other = _state(30), _state(30), _state(31)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        _step(a)
    for m in ("x", "logits", "u", "drafts"):
        a[m].copy_(other[m])
        b[m].copy_(other[m])
    graph.replay()
    _step(b)
    torch.cuda.synchronize()
    assert int(a["st"].item()) == 0 and int(b["acc"].sum()) > 0
    _same(a, b)


def test_graphs_that_share_a_workspace(gpu_lib):
    """Two captured steps on one attention workspace, one after the other, twice."""
    a, b = _state(32), _state(33)
    ref = _state(32), _state(33)
    b["ws"] = a["ws"]
    graphs = []
    for s in (a, b):
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            _step(s)
    start = [{m: s[m].clone() for m in ("ctx", "k", "v")} for s in (a, b)]
    for _ in range(2):
        for s, g, first in zip((a, b), graphs, start):
            for m in first:
                s[m].copy_(first[m])
            g.replay()
    for s, r in zip((a, b), ref):
        _step(r)
        torch.cuda.synchronize()
        _same(s, r)


def test_two_steps_at_once(gpu_lib):
    """Steps on two streams with a workspace each, many times over."""
    a, b = _state(34), _state(35)
    ref = _state(34), _state(35)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    start = [{m: s[m].clone() for m in ("ctx", "k", "v")} for s in (a, b)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, side, first in zip((a, b), streams, start):
            with torch.cuda.stream(side):
                for m in first:
                    s[m].copy_(first[m])
            _step(s, stream=side)
    torch.cuda.synchronize()
    for s, r in zip((a, b), ref):
        _step(r)
        torch.cuda.synchronize()
        _same(s, r)
        assert int(s["st"].item()) == 0


def test_a_sequence_without_drafts_among_others(gpu_lib):
    """A block of one node (nothing drafted): attention over the context and itself, the verifier's token after it."""
    c = T.cache([5, 0], [0, 0], 1, 64, 0, 40, DEV)
    par = torch.tensor([-1, -1], dtype=torch.int32, device=DEV)
    acc, nxt, new = (torch.empty(2, dtype=torch.int32, device=DEV) for _ in range(3))
    path, st = torch.empty(2, dtype=torch.int32, device=DEV), spade.status_tensor(DEV)
    tokens = torch.tensor([4, 9], dtype=torch.int32, device=DEV)
    spade.spade_tree_commit(c["k"], c["v"], c["ctx"], par, torch.empty(0, dtype=torch.int32, device=DEV), tokens, c["n"], c["cu"],
                            acc, nxt, path, new, max_k=0, status=st)
    assert acc.tolist() == [0, 0] and nxt.tolist() == [4, 9] and path.tolist() == [0, 0] and new.tolist() == [6, 1]
    assert int(st.item()) == 0


@pytest.mark.parametrize("page", [0, 64])
def test_ranges_that_begin_with_one_chunk(gpu_lib, page):
    """Many short units: a CTA's range often begins with one last chunk of a unit and goes on with another's."""
    rng = np.random.RandomState(7)
    ctx, k = rng.randint(0, 700, 96).tolist(), rng.randint(0, 3, 96).tolist()
    c = T.cache(ctx, k, 4, 128, page, 131, DEV)
    q = T.queries(c, 2, 132)
    mask = T.tree_mask(T.parents(k, "tree", 133), k, c["cu"].cpu())
    ws = gpu_lib.tree_attn_workspace(c["B"], 8, 4, 128, c["cap"], c["max_k"])
    out, lse, st = T.attention(c, q, mask, workspace=ws)
    assert int(st.item()) == 0
    T.check_attention(c, q, mask, out, lse)
    for _ in range(50):
        again, l2, st = T.attention(c, q, mask, workspace=ws)
        assert int(st.item()) == 0 and torch.equal(out, again) and torch.equal(lse, l2)
