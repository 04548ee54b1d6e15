"""The verify step's operators in 4 bits, as cases that can be timed and compared.

A verifier that holds its weights and its KV cache in 4 bits makes four kinds of call per layer and step:
the projections with 4-bit weights; the norm of every query and key head with the rotary embedding, whose
keys and values go into the 4-bit cache; the attention of the k+1 verify positions over that cache; and
the commit of the accepted positions.  Where `own` is true, run() makes these calls through the package's
public entry points; else it computes the same in elementary torch operations in 32 bits.

Numbers in 4 bits: value = scale * (code - zero) with one (scale, zero) pair of float16 per group of
neighbouring numbers, zero a whole number in 0 .. 15.  Eight neighbouring codes share a 32-bit word;
bits 4p .. 4p+3 hold number (0, 2, 4, 6, 1, 3, 5, 7)[p] of the eight.  The cache's groups are 64 dims of a
head; a group's scale spans its numbers and 0 in 15 steps.
"""
import math

import torch

own = False  # set from outside: run() calls the package's operators

DEV = "cuda"
ROPE_THETA = 500000.0
EPS = 1e-6
KV_GROUP = 64
PLACE = (0, 4, 1, 5, 2, 6, 3, 7)  # which of a word's eight 4-bit fields holds number i
MAX_SCALE = 4364.0  # 15 steps of it stay within float16

# Sizes of the verifier families: heads, head dim, hidden size.
TINY = dict(Hq=8, Hkv=8, D=64, H=512)
LLAMA2_7B = dict(Hq=32, Hkv=32, D=128, H=4096)
LLAMA3_8B = dict(Hq=32, Hkv=8, D=128, H=4096)
LONG_70B = dict(Hq=64, Hkv=8, D=128, H=8192)
GQA_40_8 = dict(Hq=40, Hkv=8, D=128, H=5120)


def _linear(R, N, K, group, residual=False):
    return dict(op="linear", R=R, N=N, K=K, group=group, residual=residual)


def _qkv_width(f):
    return (f["Hq"] + 2 * f["Hkv"]) * f["D"]


def _cache(op, f, B, ctx, k, page):
    """ctx, k: inclusive ranges over the batch; page: slots per page."""
    return dict(op=op, Hq=f["Hq"], Hkv=f["Hkv"], D=f["D"], B=B, ctx_lo=ctx[0], ctx_hi=ctx[1], k_lo=k[0], k_hi=k[1],
                page=page)


def listed():
    cases = {
        # Plain decoding of one sequence: one row against the whole projection.
        "linear_one_token": _linear(1, _qkv_width(LLAMA3_8B), LLAMA3_8B["H"], 128),
        # One interactive user's verify block, fine groups.
        "linear_7b_single": _linear(6, _qkv_width(LLAMA2_7B), LLAMA2_7B["H"], 32),
        # The output projection of four long sequences, added to the residual stream.
        "linear_70b_out": _linear(20, LONG_70B["H"], LONG_70B["Hq"] * LONG_70B["D"], 64, residual=True),
        # The verify rows of a large batch.
        "linear_ragged": _linear(389, _qkv_width(GQA_40_8), GQA_40_8["H"], 128),
        # One short sequence on a small model: latency is all there is.
        "attention_tiny": _cache("attention", TINY, 1, (256, 256), (4, 4), 64),
        # An ordinary serving batch with grouped-query heads.
        "attention_8b": _cache("attention", LLAMA3_8B, 8, (4096, 4096), (8, 8), 256),
        # Plain decoding, a token for each of many sequences of very different lengths.
        "attention_one_token": _cache("attention", GQA_40_8, 64, (0, 8192), (0, 0), 64),
        # Few very long contexts: each KV head's keys are split over many SMs.
        "attention_70b_long": _cache("attention", LONG_70B, 4, (32768, 32768), (4, 4), 128),
        # The verify blocks of a batch go into the cache.
        "norm_rope_8b": _cache("norm_rope", LLAMA3_8B, 8, (4096, 4096), (8, 8), 256),
        # Prompts go into the cache.
        "norm_rope_prompts": _cache("norm_rope", LLAMA3_8B, 8, (0, 0), (1023, 2047), 64),
        # Algorithm 1's context update after a step.
        "commit_8b": _cache("commit", LLAMA3_8B, 8, (4096, 4096), (8, 8), 256),
        "commit_ragged": _cache("commit", GQA_40_8, 64, (128, 8192), (1, 10), 64),
    }
    return [dict(name=n, **c) for n, c in cases.items()]


# ---- drawn cases ---------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges; none costs more than the largest listed one of its kind."""
    op = rng.choice(["linear", "linear", "attention", "attention", "attention", "norm_rope", "commit"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        if op == "linear":
            group = rng.choice([32, 64, 128])
            c = _linear(_log_int(rng, 1, 512), _log_int(rng, 64, 16384), group * _log_int(rng, 1, 8192 // group), group,
                        rng.random() < 0.4)
        else:
            Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
            f = dict(Hkv=Hkv, Hq=Hkv * rng.choice([1, 1, 2, 4, 4, 5, 7, 8]), D=rng.choice([64, 128, 128]))
            B = _log_int(rng, 1, 64)
            ctx_hi = _log_int(rng, 1, 32768)
            k_hi = _log_int(rng, 1, 2048) - 1 if op == "norm_rope" else rng.randint(0, 16)
            ctx_lo, k_lo = (ctx_hi, k_hi) if rng.random() < 0.5 else (rng.randint(0, ctx_hi), rng.randint(0, k_hi))
            c = _cache(op, f, B, (ctx_lo, ctx_hi), (k_lo, k_hi), 64 * rng.choice([1, 1, 2, 3, 4]))
        if _cost(c) <= most:
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _spread(lo, hi, n):
    """n lengths spread evenly over [lo, hi]."""
    return [hi] * n if lo == hi or n == 1 else [lo + round(i * (hi - lo) / (n - 1)) for i in range(n)]


def work(case):
    """What one pass cannot do without."""
    c = case
    if c["op"] == "linear":
        R, N, K = c["R"], c["N"], c["K"]
        read = N * K // 2 + 4 * N * (K // c["group"]) + 2 * R * K + (2 * R * N if c["residual"] else 0)
        return {"bytes": read + 2 * R * N, "flops": 2 * R * N * K}
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    ctx, k = _spread(c["ctx_lo"], c["ctx_hi"], B), _spread(c["k_lo"], c["k_hi"], B)
    rows = sum(k) + B
    slot = 2 * Hkv * (D // 2 + 4 * D // KV_GROUP)  # a slot's keys and values of every head
    if c["op"] == "attention":
        keys = sum(a + b + 1 for a, b in zip(ctx, k))
        pairs = sum((b + 1) * (a + 1) + b * (b + 1) // 2 for a, b in zip(ctx, k))
        return {"bytes": keys * slot + rows * Hq * (4 * D + 4), "flops": 4 * Hq * D * pairs}
    values = rows * Hkv * D * 4  # the block's slots, read back
    if c["op"] == "norm_rope":
        return {"bytes": rows * (2 * (Hq + 2 * Hkv) * D + 4 * D + 2 * Hq * D + slot) + values,
                "flops": rows * (Hq + Hkv) * D * 8}
    return {"bytes": rows * slot + values, "flops": 0}


# ---- inputs --------------------------------------------------------------------------------------
def _pack(code):
    """Codes [..., n] (whole numbers 0 .. 15) in bytes [..., n / 2]."""
    fields = code.to(torch.uint8).reshape(code.shape[:-1] + (-1, 4, 2)).transpose(-1, -2)  # even numbers first
    fields = fields.reshape(code.shape[:-1] + (code.shape[-1] // 2, 2))
    return (fields[..., 0] | (fields[..., 1] << 4)).contiguous()


def _quantise(x, group):
    """Scales, zeros [..., n / group] and codes [..., n] of numbers x [..., n], in x's precision."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    lo, hi = g.amin(-1).clamp(max=0), g.amax(-1).clamp(min=0)
    scale = ((hi - lo) * (1 / 15)).clamp(max=MAX_SCALE).to(torch.float16).to(x.dtype)
    step = torch.where(scale > 0, scale, torch.ones_like(scale))
    zero = torch.where(scale > 0, torch.round(-lo / step).clamp(0, 15), torch.zeros_like(scale))
    code = (torch.round(g / step[..., None]) + zero[..., None]).clamp(0, 15)
    return scale, zero, torch.where(scale[..., None] > 0, code, torch.zeros_like(code)).reshape(x.shape)


def _in_4_bits(x, group):
    """Numbers x [..., n] as the package's tensors: bytes [..., n / 2] and float16 pairs [..., n / group, 2]."""
    scale, zero, code = _quantise(x, group)
    return _pack(code), torch.stack((scale, zero), -1).to(torch.float16)


def _rope_table(D, positions):
    """(cos, sin) of every position and frequency, float32 [positions, D / 2, 2]."""
    freq = ROPE_THETA ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    angle = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.stack((angle.cos(), angle.sin()), -1).to(torch.float32)


def prepare(case, seed):
    """The tensors a program has before the call: inputs, 4-bit weights or pools of pages with their table, and
    the buffers it keeps."""
    c = case
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))

    def randn(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(torch.bfloat16)

    s = dict(case=c, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if c["op"] == "linear":
        R, N, K = c["R"], c["N"], c["K"]
        s["x"] = randn(R, K)
        s["codes"], s["params"] = _in_4_bits(randn(N, K, std=1 / math.sqrt(K)).float(), c["group"])
        s["residual"] = randn(R, N) if c["residual"] else None
        s["out"] = torch.empty((R, N), dtype=torch.bfloat16, device=DEV)
        return s
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    ctx = torch.tensor(_spread(c["ctx_lo"], c["ctx_hi"], B), dtype=torch.int32)[torch.randperm(B, generator=host)]
    k = torch.tensor(_spread(c["k_lo"], c["k_hi"], B), dtype=torch.int32)[torch.randperm(B, generator=host)]
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(k + 1, 0)
    R = int(cu[-1])
    s.update(R=R, max_k=c["k_hi"], ctx_lens=ctx.to(DEV), n_draft=k.to(DEV), cu_q=cu.to(DEV))
    # Pages in a shuffled order, two that nobody uses.
    n = -(-int((ctx + k).max() + 1) // page)
    s["table"] = torch.randperm(B * n + 2, generator=host)[:B * n].reshape(B, n).to(torch.int32).to(DEV)
    pool = (B * n + 2, Hkv, page)
    if c["op"] == "norm_rope":
        # A new part of the cache: slots that other sequences used before.
        for name in ("k", "v"):
            s[name + "_codes"] = torch.randint(0, 256, pool + (D // 2,), generator=gen, device=DEV, dtype=torch.uint8)
            s[name + "_params"] = torch.ones(pool + (D // KV_GROUP, 2), dtype=torch.float16, device=DEV)
        # Some heads' activations are larger; a few channels of the keys stand out.
        head = torch.exp(torch.randn((1, Hq + 2 * Hkv, 1), generator=gen, device=DEV) * 0.5)
        x = torch.randn((R, Hq + 2 * Hkv, D), generator=gen, device=DEV) * head
        s["qkv"] = x.reshape(R, -1).to(torch.bfloat16)
        s["q_norm"] = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(torch.bfloat16)
        s["k_norm"] = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(torch.bfloat16)
        s["rope"] = _rope_table(D, n * page)
        s["q"] = torch.empty((R, Hq, D), dtype=torch.bfloat16, device=DEV)
    else:
        for name in ("k", "v"):
            s[name + "_codes"], s[name + "_params"] = _in_4_bits(torch.randn(pool + (D,), generator=gen, device=DEV),
                                                                 KV_GROUP)
    if c["op"] == "attention":
        # Some heads attend broadly, others to a few keys.
        sharp = torch.exp(torch.rand((1, Hq, 1), generator=gen, device=DEV) * math.log(8.0)) * 0.5
        s["q"] = (torch.randn((R, Hq, D), generator=gen, device=DEV) * sharp).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((R, Hq), dtype=torch.float32, device=DEV)
        if own:
            import paper_2608_13076_gb300 as spade
            s["workspace"] = spade.attn_workspace(B, Hq, Hkv, D, n * page, s["max_k"], device=DEV)
    else:
        s["k_out"] = torch.empty((R, Hkv, D), dtype=torch.bfloat16, device=DEV)
        s["v_out"] = torch.empty_like(s["k_out"])
    if c["op"] == "commit":
        kept = (torch.rand(B, generator=host) * (k + 1)).floor().to(torch.int32).clamp(max=k)
        s["accepted"] = kept.to(DEV)
        s["new_ctx"] = torch.empty_like(s["ctx_lens"])
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else PLAIN[state["case"]["op"]](state)


def _run_own(s):
    import paper_2608_13076_gb300 as spade
    c = s["case"]
    if c["op"] == "linear":
        spade.spade_linear_w4(s["x"], s["codes"], s["params"], s["out"], s["residual"], status=s["status"])
        return s["out"]
    pools = (s["k_codes"], s["k_params"], s["v_codes"], s["v_params"], s["table"])
    if c["op"] == "attention":
        spade.spade_verify_attention_kv4(s["q"], *pools, s["ctx_lens"], s["n_draft"], s["cu_q"], s["out"], s["lse"],
                                         max_k=s["max_k"], workspace=s["workspace"], status=s["status"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "norm_rope":
        spade.spade_verify_qk_norm_rope_kv4(s["qkv"], s["q_norm"], s["k_norm"], s["rope"], s["q"], *pools,
                                            s["ctx_lens"], s["n_draft"], s["cu_q"], eps=EPS, max_k=s["max_k"],
                                            status=s["status"])
        first = {"q": s["q"]}
    else:
        spade.spade_kv_commit_kv4(*pools, s["ctx_lens"], s["accepted"], s["n_draft"], s["new_ctx"], status=s["status"])
        first = {"ctx": s["new_ctx"]}
    # The block's slots as the values they hold.
    spade.spade_kv_read_kv4(*pools, s["ctx_lens"], s["cu_q"], s["k_out"], s["v_out"], status=s["status"])
    return {**first, "k": s["k_out"], "v": s["v_out"]}


def _values(codes, params, dtype=torch.float32):
    """What bytes [..., n / 2] and pairs [..., n / group, 2] stand for: numbers [..., n]."""
    fields = torch.stack((codes & 15, codes >> 4), -1)
    n = 2 * codes.shape[-1]
    code = fields.reshape(codes.shape[:-1] + (n // 8, 2, 4)).transpose(-1, -2)  # even numbers first
    pair = params.to(dtype)[..., None]
    code = code.reshape(codes.shape[:-1] + (params.shape[-2], n // params.shape[-2])).to(dtype)
    return (pair[..., 0, :] * (code - pair[..., 1, :])).reshape(codes.shape[:-1] + (n,))


def _rows(s):
    """Sequence and position in the block of every row."""
    seq = torch.repeat_interleave(torch.arange(s["case"]["B"], device=DEV), (s["n_draft"] + 1).long(), output_size=s["R"])
    return seq, torch.arange(s["R"], device=DEV) - s["cu_q"][seq].long()


def _block(s, name, seq, slot):
    """The values in slots `slot` of sequences `seq`: [rows, Hkv, D]."""
    page = s["case"]["page"]
    at = s["table"][seq, slot // page].long()
    return _values(s[name + "_codes"][at, :, slot % page], s[name + "_params"][at, :, slot % page])


def _plain_linear(s):
    y = s["x"].float() @ _values(s["codes"], s["params"]).T
    return (y + s["residual"].float() if s["residual"] is not None else y).to(torch.bfloat16)


def _plain_attention(s):
    c = s["case"]
    B, Hq, Hkv, D, R = c["B"], c["Hq"], c["Hkv"], c["D"], s["R"]
    seq, i = _rows(s)
    wide = s["max_k"] + 1
    q = torch.zeros((B, wide, Hq, D), device=DEV)
    q[seq, i] = s["q"].float()
    q = q.reshape(B, wide, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)

    def keys(name):
        v = _values(s[name + "_codes"][s["table"].long()], s[name + "_params"][s["table"].long()])
        return v.transpose(1, 2).reshape(B, Hkv, -1, D)

    score = (q @ keys("k").transpose(2, 3)) / math.sqrt(D)
    score = score.reshape(B, Hkv, Hq // Hkv, wide, -1)
    last = s["ctx_lens"].long()[:, None] + torch.arange(wide, device=DEV)
    seen = torch.arange(score.shape[-1], device=DEV) <= last[..., None]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    out = (p.reshape(B, Hkv, -1, p.shape[-1]) @ keys("v")).reshape(B, Hkv, Hq // Hkv, wide, D) / total
    lse = (top + torch.log(total))[..., 0]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, wide, Hq, D)[seq, i]
    return {"out": out.to(torch.bfloat16), "lse": lse.permute(0, 3, 1, 2).reshape(B, wide, Hq)[seq, i]}


def _plain_norm_rope(s):
    c = s["case"]
    Hq, Hkv, D, R = c["Hq"], c["Hkv"], c["D"], s["R"]
    seq, i = _rows(s)
    q, k, v = s["qkv"].float().reshape(R, -1, D).split((Hq, Hkv, Hkv), 1)
    turn = s["rope"][s["ctx_lens"][seq].long() + i][:, None]

    def turned(x, weight):
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat((a * turn[..., 0] - b * turn[..., 1], b * turn[..., 0] + a * turn[..., 1]), -1)

    def held(x):
        scale, zero, code = _quantise(x, KV_GROUP)
        code = code.reshape(R, Hkv, -1, KV_GROUP)
        return (scale[..., None] * (code - zero[..., None])).reshape(R, Hkv, D).to(torch.bfloat16)

    return {"q": turned(q, s["q_norm"]).to(torch.bfloat16), "k": held(turned(k, s["k_norm"])), "v": held(v)}


def _plain_commit(s):
    seq, i = _rows(s)
    slot = s["ctx_lens"][seq].long() + i
    kept = (i <= s["accepted"][seq])[:, None, None]
    return {"ctx": s["ctx_lens"] + s["accepted"] + 1,
            "k": torch.where(kept, _block(s, "k", seq, slot), 0.0).to(torch.bfloat16),
            "v": torch.where(kept, _block(s, "v", seq, slot), 0.0).to(torch.bfloat16)}


PLAIN = {"linear": _plain_linear, "attention": _plain_attention, "norm_rope": _plain_norm_rope, "commit": _plain_commit}


# ---- the definition in 64 bits ---------------------------------------------------------------------
def _numbers(codes, params):
    """Values of 4-bit numbers, code by code, in 64 bits."""
    n = 2 * codes.shape[-1]
    group = n // params.shape[-2]
    out = torch.empty(codes.shape[:-1] + (n,), dtype=torch.float64, device=codes.device)
    for i in range(8):
        byte, high = divmod(PLACE[i], 2)
        c = codes[..., byte::4]
        out[..., i::8] = (c >> 4 if high else c & 15).double()
    scale, zero = params[..., 0].double(), params[..., 1].double()
    return (out - zero.repeat_interleave(group, -1)) * scale.repeat_interleave(group, -1)


def _held_exactly(x):
    """What the cache holds of numbers x [..., D] in 64 bits."""
    g = x.reshape(*x.shape[:-1], -1, KV_GROUP)
    lo, hi = torch.minimum(g.amin(-1, True), g.new_zeros(())), torch.maximum(g.amax(-1, True), g.new_zeros(()))
    scale = torch.minimum((hi - lo) / 15, g.new_tensor(MAX_SCALE)).half().double()
    none = scale == 0
    by = torch.where(none, torch.ones_like(scale), scale)
    zero = torch.clamp(torch.round(-lo / by), 0, 15)
    value = scale * (torch.clamp(torch.round(g / by) + zero, 0, 15) - zero)
    return torch.where(none, torch.zeros_like(value), value).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        y = s["x"].double() @ _numbers(s["codes"], s["params"]).T
        return y if s["residual"] is None else y + s["residual"].double()
    B, Hq, Hkv, D, page = (case[n] for n in ("B", "Hq", "Hkv", "D", "page"))
    ctx, k, cu = s["ctx_lens"].tolist(), s["n_draft"].tolist(), s["cu_q"].tolist()
    parts = []
    for b in range(B):
        at, n = s["table"][b].long(), ctx[b] + k[b] + 1
        rows = slice(cu[b], cu[b + 1])
        if case["op"] == "norm_rope":
            x = s["qkv"][rows].double().reshape(k[b] + 1, Hq + 2 * Hkv, D)
            norm = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            turn = torch.view_as_complex(s["rope"][ctx[b]:n].double())[:, None]

            def turned(y):
                z = torch.complex(y[..., :D // 2], y[..., D // 2:]) * turn
                return torch.cat((z.real, z.imag), -1)

            parts.append({"q": turned(norm[:, :Hq] * s["q_norm"].double()),
                          "k": _held_exactly(turned(norm[:, Hq:Hq + Hkv] * s["k_norm"].double())),
                          "v": _held_exactly(x[:, Hq + Hkv:])})
            continue
        # The sequence's pages, in order, as [slots, Hkv, D].
        K, V = (_numbers(s[m + "_codes"][at], s[m + "_params"][at]).transpose(1, 2).reshape(-1, Hkv, D)[:n] for m in "kv")
        if case["op"] == "commit":
            keep = int(s["accepted"][b]) + 1
            new = []
            for x in (K, V):
                x = x[ctx[b]:].clone()
                x[keep:] = 0
                new.append(x)
            parts.append({"ctx": torch.tensor([ctx[b] + keep], dtype=torch.int32, device=DEV), "k": new[0], "v": new[1]})
            continue
        q = s["q"][rows].double().reshape(k[b] + 1, Hkv, Hq // Hkv, D)
        score = torch.einsum("ihgd,shd->ihgs", q, K) / math.sqrt(D)
        for i in range(k[b] + 1):
            score[i, :, :, ctx[b] + i + 1:] = -math.inf
        out = torch.einsum("ihgs,shd->ihgd", torch.softmax(score, -1), V)
        parts.append({"out": out.reshape(k[b] + 1, Hq, D), "lse": torch.logsumexp(score, -1).reshape(k[b] + 1, Hq)})
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
