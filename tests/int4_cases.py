"""Seeded inputs of the 4-bit verify step's tests: paged caches with stale and poisoned slots around the live ones."""
import numpy as np
import torch

import paper_2608_13076_gb300 as spade
from paper_2608_13076_gb300 import int4


def lengths(ctx, k):
    ctx, k = torch.tensor(ctx, dtype=torch.int32), torch.tensor(k, dtype=torch.int32)
    cu = torch.zeros(len(ctx) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(k + 1, 0)
    return ctx, k, cu


def cache(ctx, k, Hkv, D, page, seed, dev, scale=1.0, spare=2, poison=True):
    """A filled paged cache: dict(pools, table, ctx, k, cu, ...).  Slots past ctx + k hold NaN scales
    and arbitrary codes, as do the spare pages."""
    gen = torch.Generator().manual_seed(seed)
    ctx, k, cu = lengths(ctx, k)
    B = len(ctx)
    n = max(1, -(-int((ctx + k).max() + 1) // page))
    table = torch.randperm(B * n + spare, generator=gen)[:B * n].reshape(B, n).to(torch.int32)
    pools = []
    for _ in range(2):
        x = torch.randn((B * n + spare, Hkv, page, D), generator=gen) * scale
        codes, params = int4.quantize(x, 64)
        if poison:
            live = torch.zeros((B * n + spare, page), dtype=torch.bool)
            for b in range(B):
                for s in range(int(ctx[b] + k[b]) + 1):
                    live[int(table[b, s // page]), s % page] = True
            params[~live[:, None].expand(-1, Hkv, -1)] = float("nan")
        pools += [codes.to(dev), params.to(dev)]
    return dict(pools=pools, table=table.to(dev), ctx=ctx.to(dev), k=k.to(dev), cu=cu.to(dev), B=B, R=int(cu[-1]),
                max_k=int(k.max()), Hkv=Hkv, D=D, page=page, max_pages=n, gen=gen)


def queries(c, G, seed, sharp=1.0):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn((c["R"], c["Hkv"] * G, c["D"]), generator=gen) * sharp
    return q.to(torch.bfloat16).to(c["table"].device)


def attention(c, q, max_k=None, workspace=None, stream=None, lse=True):
    dev = q.device
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device=dev) if lse else None
    max_k = c["max_k"] if max_k is None else max_k
    if workspace is None:
        workspace = spade.attn_workspace(c["B"], q.shape[1], c["Hkv"], c["D"], c["max_pages"] * c["page"], max_k, device=dev)
    st = spade.status_tensor(dev)
    spade.spade_verify_attention_kv4(q, *c["pools"], c["table"], c["ctx"], c["k"], c["cu"], out, lse, max_k=max_k,
                                     workspace=workspace, status=st, stream=stream)
    return out, lse, st


def np64(t):
    t = t.detach().cpu()
    return t.float().numpy() if t.dtype == torch.bfloat16 else t.numpy()


def arrays(c):
    return [np64(t) for t in c["pools"]], np64(c["table"]), np64(c["ctx"]), np64(c["k"]), np64(c["cu"])


def check_attention(c, q, out, lse):
    """Every element against float64.  What the kernels may lose, from their roundings: scores are fp32 sums of D
    products (error at most D 2^-23 of the sum of their sizes); weights and values may be held in float16 (2^-11
    each, weights below 2^-20 of the largest lose up to 2^-32 of it); sums in fp32; the result in bf16 (2^-8)."""
    from oracle import int4_oracle as O
    pools, table, ctx, k, cu = arrays(c)
    ref, rlse, mass, smass = O.attention(np64(q), pools, table, ctx, k, cu)
    n = int((ctx + k).max()) + 1
    ds = (c["D"] * 2.0 ** -23 * smass + 2.0 ** -20)[..., None]
    vmax = np.abs(ref).max() + mass.max()
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + 2 * ds + n * 2.0 ** -24) * mass + n * 2.0 ** -31 * vmax
    got = np64(out).astype(np.float64)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())
    if lse is not None:
        tl = ds[..., 0] + 2.0 ** -20 * (1 + np.abs(rlse)) + n * 2.0 ** -24
        assert (np.abs(np64(lse) - rlse) <= tl).all(), float((np.abs(np64(lse) - rlse) / tl).max())
