"""A multi-step speculative-decoding loop (Algorithm 1) on the GPU with a toy verifier.

The cloud verifier is a small random one-layer decoder whose verify step runs
through this library: the QKV projection with rotary embedding writes the
verify block's keys and values into the cache (spade_verify_qkv_rope), the
verify attention reads them (spade_verify_attention), the output projection
adds the attention to the residual stream (x_{l+1} = x_l + f_l(x_l), Sec.
III-A; a plain bf16 matmul), and the LM head with the fused accept test,
residual sampling and KV commit closes the step (spade_verify_accept_commit).
The edge drafter proposes d tokens per round from a cheap model whose logits
are the verifier's without the attention term (its residual path only), so
its q is correlated with the verifier's p, as a real draft model's is.

Each round: the drafter proposes d tokens (greedy: its argmax; stochastic: a
draw from q, which is sent along), the verifier scores the d + 1 positions in
one call, and every sequence appends its accepted drafts plus the correction
or bonus token (Algorithm 1's cloud step and context update).  The loop runs
until each sequence has produced `max_new` tokens or its end-of-sequence
token, and reports verifier calls against tokens, the quantity the paper's
cloud-call reduction is about (Sec. IV).

ToyVerifierInt4 is the same model with its projections' weights and its KV cache in
4 bits: spade_linear_w4 for the projections (the output projection adds the residual),
spade_verify_qk_norm_rope_kv4 into a paged cache, spade_verify_attention_kv4 over it,
the LM head without a commit and spade_kv_commit_kv4.

ToyVerifierTree is a decoder of several such layers whose blocks are trees of drafts
(speculative_tree_decode): spade_tree_layout, spade_verify_rope and
spade_verify_attention_tree in every layer on paged caches, spade_sample for the
verifier's token at every node, spade_tree_commit for the path that is kept.  A prompt
is a tree without branches and goes the same way.

This is a toy model for exercising and measuring the verify path end to end;
it is not a trained model.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import (accept_workspace, attn_workspace, int4, qkv_workspace, rope, spade_kv_commit_kv4, spade_linear_w4,
               spade_sample, spade_tree_commit_paged, spade_tree_layout, spade_verify_accept, spade_verify_accept_commit,
               spade_verify_accept_sampling, spade_verify_attention, spade_verify_attention_kv4,
               spade_verify_attention_tree_paged, spade_verify_qk_norm_rope_kv4, spade_verify_qkv_rope,
               spade_verify_rope_paged, status_tensor, tree_attn_workspace)

GREEDY = 0
STOCHASTIC = 1


@dataclass
class ToyConfig:
    V: int = 2048        # vocabulary (token V - 1 is the end-of-sequence token)
    H: int = 512         # hidden size
    Hq: int = 8          # query heads
    Hkv: int = 2         # key/value heads
    D: int = 64          # head dimension
    rope_theta: float = 10000.0
    logit_scale: float = 4.0  # sharpens the toy distributions (logits ~ N(0, scale^2))


class ToyVerifier:
    """Random one-layer decoder (embedding, attention layer, LM head) with a KV cache of
    `cap` slots for each of `B` sequences, on `device`; weights drawn on the CPU from `seed`."""

    def __init__(self, cfg: ToyConfig, B: int, cap: int, seed: int, device):
        self.cfg, self.B, self.cap = cfg, B, cap
        dev = torch.device(device)
        g = torch.Generator().manual_seed(seed)

        def normal(shape, std):
            return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).to(dev)

        c = cfg
        self.emb = normal((c.V, c.H), 1.0)
        self.w_qkv = normal(((c.Hq + 2 * c.Hkv) * c.D, c.H), 1.0 / math.sqrt(c.H))
        self.w_o = normal((c.H, c.Hq * c.D), 1.0 / math.sqrt(c.Hq * c.D))
        self.w_lm = normal((c.V, c.H), c.logit_scale / math.sqrt(c.H))
        self.ctx = torch.zeros(B, dtype=torch.int32, device=dev)
        self.status = status_tensor(dev)
        self.device = dev
        self._make_cache()

    def _make_cache(self):
        c = self.cfg
        self.k_cache = torch.zeros((self.B, c.Hkv, self.cap, c.D), dtype=torch.bfloat16, device=self.device)
        self.v_cache = torch.zeros_like(self.k_cache)

    def draft_logits(self, tokens):
        """The drafter's logits after `tokens` [n]: the verifier's residual path without its
        attention term, fp32 [n, V]."""
        return self.emb[tokens].float() @ self.w_lm.float().t()

    def write_prefix(self, tokens, ctx, kd, cu_q, max_k):
        """K/V of prompt tokens (no output needed: one layer)."""
        x = self.emb[tokens].contiguous()
        q = torch.empty((x.shape[0], self.cfg.Hq, self.cfg.D), dtype=torch.bfloat16, device=self.device)
        spade_verify_qkv_rope(x, self.w_qkv, ctx, kd, cu_q, q, self.k_cache, self.v_cache, Hq=self.cfg.Hq,
                              Hkv=self.cfg.Hkv, rope_theta=self.cfg.rope_theta, max_k=max_k,
                              workspace=qkv_workspace(x.shape[0], self.cfg.Hq, self.cfg.Hkv, self.cfg.D,
                                                      device=self.device), status=self.status)

    def verify(self, tokens, kd, cu_q, drafts, draft_probs, uniforms, mode, max_k, temperature=None, top_p=None):
        """One verify call over the blocks (row cu_q[b] + i holds token i of sequence b's
        block, position ctx_b + i): returns (accepted_len, next_token); the cache and ctx
        are committed (accepted slots kept, rejected ones cleared, ctx += a + 1).  With
        ``temperature`` / ``top_p`` ([B] float32) the verifier's p is softmax(l / T) cut to
        its nucleus."""
        c = self.cfg
        R = tokens.numel()
        x = self.emb[tokens].contiguous()
        q = torch.empty((R, c.Hq, c.D), dtype=torch.bfloat16, device=self.device)
        spade_verify_qkv_rope(x, self.w_qkv, self.ctx, kd, cu_q, q, self.k_cache, self.v_cache, Hq=c.Hq,
                              Hkv=c.Hkv, rope_theta=c.rope_theta, max_k=max_k,
                              workspace=qkv_workspace(R, c.Hq, c.Hkv, c.D, device=self.device), status=self.status)
        out = torch.empty_like(q)
        ws = attn_workspace(self.B, c.Hq, c.Hkv, c.D, self.cap, max_k, device=self.device)
        spade_verify_attention(q, self.k_cache, self.v_cache, self.ctx, kd, cu_q, out, None, max_k=max_k,
                               workspace=ws, status=self.status)
        hidden = (x.float() + out.reshape(R, c.Hq * c.D).float() @ self.w_o.float().t()).to(torch.bfloat16)
        acc = torch.empty(self.B, dtype=torch.int32, device=self.device)
        tok = torch.empty_like(acc)
        wsa = accept_workspace(self.B, R, c.H, c.V, device=self.device)
        if temperature is None and top_p is None:
            spade_verify_accept_commit(hidden.contiguous(), self.w_lm, drafts, draft_probs, uniforms, mode, cu_q,
                                       kd, acc, tok, self.k_cache, self.v_cache, self.ctx, workspace=wsa,
                                       status=self.status)
        else:
            spade_verify_accept_sampling(hidden.contiguous(), self.w_lm, drafts, draft_probs, uniforms, mode, cu_q,
                                         kd, acc, tok, workspace=wsa, status=self.status, temperature=temperature,
                                         top_p=top_p, k_cache=self.k_cache, v_cache=self.v_cache,
                                         ctx_lens=self.ctx)
        self.last_hidden = hidden
        return acc, tok


class ToyVerifierInt4(ToyVerifier):
    """ToyVerifier's decoder with 4-bit projections (groups of `group` along the inputs), norms on
    the query and key heads, and a paged 4-bit cache in pages of `page` slots."""

    def __init__(self, cfg: ToyConfig, B: int, cap: int, seed: int, device, page: int = 64, group: int = 64):
        self.page = page
        super().__init__(cfg, B, cap, seed, device)
        c, dev = cfg, self.device
        self.w_qkv, self.w_o = (int4.quantize(w, group) for w in (self.w_qkv, self.w_o))
        self.q_norm = torch.ones(c.D, dtype=torch.bfloat16, device=dev)
        self.k_norm = torch.ones_like(self.q_norm)
        self.rope = int4.rope_table(c.rope_theta, c.D, self.table.shape[1] * page, device=dev)

    def _make_cache(self):
        # Pages dealt to the sequences in turn, as a serving pool would end up.
        B, max_pages = self.B, -(-self.cap // self.page)
        self.pools = int4.kv4_pools(B * max_pages, self.cfg.Hkv, self.page, self.cfg.D, device=self.device)
        self.table = torch.arange(B * max_pages, dtype=torch.int32).reshape(max_pages, B).t().contiguous().to(self.device)

    def _heads(self, x, ctx, kd, cu_q, max_k):
        """Query heads of rows x; their keys and values go into the cache at ctx + i."""
        c, R = self.cfg, x.shape[0]
        qkv = torch.empty((R, (c.Hq + 2 * c.Hkv) * c.D), dtype=torch.bfloat16, device=self.device)
        spade_linear_w4(x, *self.w_qkv, qkv, status=self.status)
        q = torch.empty((R, c.Hq, c.D), dtype=torch.bfloat16, device=self.device)
        return spade_verify_qk_norm_rope_kv4(qkv, self.q_norm, self.k_norm, self.rope, q, *self.pools, self.table, ctx, kd,
                                             cu_q, eps=1e-6, max_k=max_k, status=self.status)

    def write_prefix(self, tokens, ctx, kd, cu_q, max_k):
        self._heads(self.emb[tokens].contiguous(), ctx, kd, cu_q, max_k)

    def verify(self, tokens, kd, cu_q, drafts, draft_probs, uniforms, mode, max_k, temperature=None, top_p=None):
        c, R = self.cfg, tokens.numel()
        x = self.emb[tokens].contiguous()
        q = self._heads(x, self.ctx, kd, cu_q, max_k)
        out = torch.empty_like(q)
        slots = self.table.shape[1] * self.page
        ws = attn_workspace(self.B, c.Hq, c.Hkv, c.D, slots, max_k, device=self.device)
        spade_verify_attention_kv4(q, *self.pools, self.table, self.ctx, kd, cu_q, out, None, max_k=max_k, workspace=ws,
                                   status=self.status)
        hidden = torch.empty_like(x)
        spade_linear_w4(out.reshape(R, c.Hq * c.D), *self.w_o, hidden, x, status=self.status)
        acc = torch.empty(self.B, dtype=torch.int32, device=self.device)
        tok = torch.empty_like(acc)
        wsa = accept_workspace(self.B, R, c.H, c.V, device=self.device)
        if temperature is None and top_p is None:
            spade_verify_accept(hidden, self.w_lm, drafts, draft_probs, uniforms, mode, cu_q, kd, acc, tok, workspace=wsa,
                                status=self.status)
        else:
            spade_verify_accept_sampling(hidden, self.w_lm, drafts, draft_probs, uniforms, mode, cu_q, kd, acc, tok,
                                         workspace=wsa, status=self.status, temperature=temperature, top_p=top_p)
        spade_kv_commit_kv4(*self.pools, self.table, self.ctx, acc, kd, self.ctx, status=self.status)
        self.last_hidden = hidden
        return acc, tok


class ToyVerifierTree(ToyVerifier):
    """A decoder of `layers` attention layers over paged caches in pages of `page` slots, whose verify blocks are
    trees.  ``scaling``: how the rotary frequencies are stretched (arguments of rope.inv_freq); ``mscale``: the factor of
    the turned dims, where the model has one (rope.attention_scale)."""

    def __init__(self, cfg: ToyConfig, B: int, cap: int, seed: int, device, layers: int = 2, page: int = 64, scaling=None,
                 mscale: float = 1.0):
        self.layers, self.page = layers, page
        super().__init__(cfg, B, cap, seed, device)
        c = cfg
        g = torch.Generator().manual_seed(seed + 1)
        for name, std in (("w_qkv", 1.0 / math.sqrt(c.H)), ("w_o", 1.0 / math.sqrt(c.Hq * c.D))):
            first = getattr(self, name)
            more = [(torch.randn(first.shape, generator=g) * std).to(first) for _ in range(layers - 1)]
            setattr(self, name, torch.stack([first] + more))
        self.inv_freq = rope.inv_freq(c.rope_theta, c.D, device=self.device, **(scaling or {}))
        self.mscale = mscale
        self.workspace = None

    def _make_cache(self):
        # Pages dealt to the sequences in turn, as a serving pool would end up.
        B, max_pages = self.B, -(-self.cap // self.page)
        shape = (self.layers, B * max_pages, self.cfg.Hkv, self.page, self.cfg.D)
        self.k_pools = torch.zeros(shape, dtype=torch.bfloat16, device=self.device)
        self.v_pools = torch.zeros_like(self.k_pools)
        self.table = torch.arange(B * max_pages, dtype=torch.int32).reshape(max_pages, B).t().contiguous().to(self.device)

    def _workspace(self):
        # One for blocks of every size, as its own depends on the head dim alone.
        c = self.cfg
        if self.workspace is None:
            self.workspace = tree_attn_workspace(self.B, c.Hq, c.Hkv, c.D, self.table.shape[1] * self.page, 0,
                                                 device=self.device)
        return self.workspace

    def _hidden(self, tokens, parents, kd, cu_q, max_k):
        """The last layer's output at every node; the nodes' keys and values are in the caches' slots from ctx on."""
        c, R = self.cfg, tokens.numel()
        pos = torch.empty(R, dtype=torch.int32, device=self.device)
        mask = torch.empty((R, max_k // 32 + 1), dtype=torch.int32, device=self.device)
        spade_tree_layout(parents, self.ctx, kd, cu_q, pos, mask, max_k=max_k, status=self.status)
        x = self.emb[tokens]
        q = torch.empty((R, c.Hq, c.D), dtype=torch.bfloat16, device=self.device)
        out = torch.empty_like(q)
        for i in range(self.layers):
            kv = self.k_pools[i], self.v_pools[i]
            spade_verify_rope_paged(x @ self.w_qkv[i].t(), self.inv_freq, pos, self.table, self.ctx, kd, cu_q, q, *kv,
                                    mscale=self.mscale, max_k=max_k, status=self.status)
            spade_verify_attention_tree_paged(q, *kv, self.table, self.ctx, kd, cu_q, mask, out, max_k=max_k,
                                              workspace=self._workspace(), status=self.status)
            x = (x.float() + out.reshape(R, c.Hq * c.D).float() @ self.w_o[i].float().t()).to(torch.bfloat16)
        return x

    def write_prefix(self, tokens, ctx, kd, cu_q, max_k):
        """K/V of prompt tokens, each prompt a chain."""
        lens = (kd + 1).long()
        parents = torch.arange(tokens.numel(), device=self.device) - torch.repeat_interleave(cu_q[:-1].long(), lens) - 1
        self._hidden(tokens, parents.to(torch.int32), kd, cu_q, max_k)

    def verify(self, *args, **kwargs):
        raise TypeError("ToyVerifierTree verifies trees: use speculative_tree_decode (a chain is a tree of widths 1)")

    def verify_tree(self, tokens, parents, kd, cu_q, drafts, uniforms, max_k, **options):
        """One verify call over the trees (row cu_q[b] + i holds node i's token): (accepted_len, next_token, path); the
        caches keep the path, ctx += a + 1.  ``options``: spade_sample's."""
        R = tokens.numel()
        self.last_hidden = self._hidden(tokens, parents, kd, cu_q, max_k)
        logits = self.last_hidden.float() @ self.w_lm.float().t()
        target = torch.empty(R, dtype=torch.int32, device=self.device)
        spade_sample(logits, uniforms, target, status=self.status, **options)
        acc = torch.empty(self.B, dtype=torch.int32, device=self.device)
        tok, path = torch.empty_like(acc), torch.empty_like(target)
        spade_tree_commit_paged(self.k_pools, self.v_pools, self.table, self.ctx, parents, drafts, target, kd, cu_q, acc,
                                tok, path, self.ctx, max_k=max_k, status=self.status)
        return acc, tok, path


def tree_of(widths):
    """Parents of a tree whose nodes of depth t have widths[t] children, level by level, and its levels' first nodes."""
    parents, first = [-1], [0]
    level = [0]
    for w in widths:
        first.append(len(parents))
        parents += [i for i in level for _ in range(w)]
        level = range(first[-1], len(parents))
    return parents, first


@dataclass
class LoopResult:
    tokens: list          # per sequence: the generated tokens after the prompt (<= max_new)
    calls: int            # verifier calls of the whole batch
    calls_per_seq: list   # verifier calls until each sequence was done
    drafted: int          # drafts proposed for sequences not yet done
    accepted: int         # of those, drafts the verifier accepted
    margins: list         # with record_margins and d = 0: per sequence, the top-2 logit gap of each token


def speculative_decode(ver: ToyVerifier, prompts, d: int, max_new: int, mode: int = GREEDY, seed: int = 0,
                       eos: int | None = None, record_margins: bool = False, temperature: float | None = None,
                       top_p: float | None = None) -> LoopResult:
    """Algorithm 1 for a batch of prompts (each at least 2 tokens): rounds of d drafts and one
    verifier call, until every sequence has max_new tokens or has emitted `eos` (default
    V - 1).  d = 0 is plain decoding with the verifier alone.  Stochastic mode draws the
    drafts from q = softmax(drafter logits) and the uniforms from a CPU generator seeded
    with `seed`; `temperature` and `top_p` (one value for every sequence) shape the
    verifier's p.  The verifier's cache must hold every prompt plus max_new * (d + 1) + d + 1
    slots (sequences that are done keep stepping with the batch)."""
    B, cfg, dev = ver.B, ver.cfg, ver.device
    eos = cfg.V - 1 if eos is None else eos
    assert len(prompts) == B and all(len(p) >= 2 for p in prompts)
    need = max(len(p) for p in prompts) + max_new * (d + 1) + d + 1
    if need > ver.cap:
        raise ValueError(f"cache of {ver.cap} slots is too small; this loop needs {need}")
    gen = torch.Generator().manual_seed(seed)
    # Prefill: the prompt tokens before the last one go into the cache.
    pre = [torch.tensor(p[:-1], dtype=torch.long) for p in prompts]
    lens = torch.tensor([len(x) for x in pre], dtype=torch.int32)
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(lens, 0)
    ver.ctx.zero_()
    ver.write_prefix(torch.cat(pre).to(dev), ver.ctx, (lens - 1).to(dev), cu.to(dev), int(lens.max()) - 1)
    ver.ctx.copy_(lens.to(dev))
    last = torch.tensor([p[-1] for p in prompts], dtype=torch.long, device=dev)
    mode_t = torch.full((B,), mode, dtype=torch.int32, device=dev)
    temp_t = None if temperature is None else torch.full((B,), temperature, dtype=torch.float32, device=dev)
    top_p_t = None if top_p is None else torch.full((B,), top_p, dtype=torch.float32, device=dev)
    kd = torch.full((B,), d, dtype=torch.int32, device=dev)
    cu_q = (torch.arange(B + 1, dtype=torch.int32) * (d + 1)).to(dev)
    out = [[] for _ in range(B)]
    margins = [[] for _ in range(B)]
    done = [False] * B
    calls, calls_per_seq, drafted, accepted = 0, [0] * B, 0, 0
    while not all(done):
        cur = last
        drafts, qrows = [], []
        for _ in range(d):
            lg = ver.draft_logits(cur)
            if mode == GREEDY:
                nxt = lg.argmax(-1)
            else:
                qd = torch.softmax(lg, dim=-1)
                nxt = torch.multinomial(qd.cpu(), 1, generator=gen).flatten().to(dev)
                qrows.append(qd)
            drafts.append(nxt)
            cur = nxt
        rows = torch.stack([last] + drafts, dim=1)  # [B, d + 1]: last accepted token, then the drafts
        dr = torch.stack(drafts, dim=1).reshape(-1).to(torch.int32) if d else \
            torch.empty(0, dtype=torch.int32, device=dev)
        qp = torch.stack(qrows, dim=1).reshape(B * d, cfg.V).contiguous() if (d and mode == STOCHASTIC) else None
        u = torch.rand(B * (d + 1), generator=gen).to(dev)
        acc, tok = ver.verify(rows.reshape(-1), kd, cu_q, dr, qp, u, mode_t, d, temperature=temp_t, top_p=top_p_t)
        calls += 1
        acc_l, tok_l = acc.tolist(), tok.tolist()
        gap_l = None
        if record_margins and d == 0:
            # Diagnostic beside the decision: the top-2 gap of the row that emitted each token.
            top = (ver.last_hidden.float() @ ver.w_lm.float().t()).topk(2, dim=-1).values
            gap_l = (top[:, 0] - top[:, 1]).tolist()
        dr_l = rows[:, 1:].tolist()
        for b in range(B):
            if not done[b]:
                calls_per_seq[b] += 1
                drafted += d
                accepted += acc_l[b]
                for t in dr_l[b][:acc_l[b]] + [tok_l[b]]:
                    if len(out[b]) < max_new and not (out[b] and out[b][-1] == eos):
                        out[b].append(t)
                        if gap_l is not None:
                            margins[b].append(gap_l[b])
                done[b] = len(out[b]) >= max_new or (bool(out[b]) and out[b][-1] == eos)
        last = tok.to(torch.long)
    if int(ver.status.item()) & ~0x8:
        raise RuntimeError(f"device status {int(ver.status.item())} in the decoding loop")
    return LoopResult(out, calls, calls_per_seq, drafted, accepted, margins)


def speculative_tree_decode(ver: ToyVerifierTree, prompts, widths, max_new: int, mode: int = GREEDY, seed: int = 0,
                            eos: int | None = None, record_margins: bool = False, temperature: float = 1.0, top_k: int = 0,
                            top_p: float = 1.0, min_p: float = 0.0) -> LoopResult:
    """speculative_decode with trees of drafts: a node of depth t has widths[t] children, the drafter's likeliest tokens
    after it (greedy) or draws from its distribution (stochastic: the children of a node may repeat).  The verifier's
    token at a node is its argmax (greedy) or a draw under the options.  widths () is plain decoding.  The cache must hold
    every prompt plus (max_new - 1) * (len(widths) + 1) slots and one block."""
    if not isinstance(ver, ToyVerifierTree):
        raise TypeError("speculative_tree_decode needs a ToyVerifierTree")
    B, cfg, dev = ver.B, ver.cfg, ver.device
    eos = cfg.V - 1 if eos is None else eos
    parents, first = tree_of(widths)
    n = len(parents)
    if len(prompts) != B or not all(len(p) >= 2 for p in prompts):
        raise ValueError(f"{B} prompts of two tokens and more are needed")
    need = max(len(p) for p in prompts) - 1 + (max_new - 1) * (len(widths) + 1) + n
    if need > ver.cap:
        raise ValueError(f"cache of {ver.cap} slots is too small; this loop needs {need}")
    gen = torch.Generator().manual_seed(seed)
    pre = [torch.tensor(p[:-1], dtype=torch.long) for p in prompts]
    lens = torch.tensor([len(x) for x in pre], dtype=torch.int32)
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(lens, 0)
    ver.ctx.zero_()
    ver.write_prefix(torch.cat(pre).to(dev), ver.ctx, (lens - 1).to(dev), cu.to(dev), int(lens.max()) - 1)
    ver.ctx.copy_(lens.to(dev))
    kd = torch.full((B,), n - 1, dtype=torch.int32, device=dev)
    cu_q = (torch.arange(B + 1, dtype=torch.int32) * n).to(dev)
    par = torch.tensor(parents * B, dtype=torch.int32, device=dev)
    per_row = lambda x, dtype: torch.full((B * n,), x, dtype=dtype, device=dev)
    options = dict(temperature=per_row(0.0 if mode == GREEDY else temperature, torch.float32))
    if mode != GREEDY:
        options.update(top_k=per_row(top_k, torch.int32), top_p=per_row(top_p, torch.float32),
                       min_p=per_row(min_p, torch.float32))
    nodes = torch.empty((B, n), dtype=torch.long, device=dev)
    nodes[:, 0] = torch.tensor([p[-1] for p in prompts], dtype=torch.long)
    out = [[] for _ in range(B)]
    margins = [[] for _ in range(B)]
    done = [False] * B
    calls, calls_per_seq, drafted, accepted = 0, [0] * B, 0, 0
    while not all(done):
        for t, w in enumerate(widths):
            f, m = first[t], first[t + 1] - first[t]
            lg = ver.draft_logits(nodes[:, f:f + m].reshape(-1))
            if mode == GREEDY:
                kids = lg.topk(w, dim=-1).indices
            else:
                kids = torch.empty(B * m * w, dtype=torch.int32, device=dev)
                spade_sample(lg.repeat_interleave(w, 0), torch.rand(B * m * w, generator=gen).to(dev), kids,
                             status=ver.status)
            nodes[:, first[t + 1]:first[t + 1] + m * w] = kids.reshape(B, m * w)
        drafts = nodes[:, 1:].reshape(-1).to(torch.int32)
        u = torch.rand(B * n, generator=gen).to(dev)
        acc, tok, path = ver.verify_tree(nodes.reshape(-1), par, kd, cu_q, drafts, u, n - 1, **options)
        calls += 1
        acc_l, tok_l, path_l, nodes_l = acc.tolist(), tok.tolist(), path.reshape(B, n).tolist(), nodes.tolist()
        gap_l = None
        if record_margins and n == 1:
            top = (ver.last_hidden.float() @ ver.w_lm.float().t()).topk(2, dim=-1).values
            gap_l = (top[:, 0] - top[:, 1]).tolist()
        for b in range(B):
            if not done[b]:
                calls_per_seq[b] += 1
                drafted += n - 1
                accepted += acc_l[b]
                for t in [nodes_l[b][j] for j in path_l[b][1:acc_l[b] + 1]] + [tok_l[b]]:
                    if len(out[b]) < max_new and not (out[b] and out[b][-1] == eos):
                        out[b].append(t)
                        if gap_l is not None:
                            margins[b].append(gap_l[b])
                done[b] = len(out[b]) >= max_new or (bool(out[b]) and out[b][-1] == eos)
        nodes[:, 0] = tok.long()
    if int(ver.status.item()):
        raise RuntimeError(f"device status {int(ver.status.item())} in the decoding loop")
    return LoopResult(out, calls, calls_per_seq, drafted, accepted, margins)
