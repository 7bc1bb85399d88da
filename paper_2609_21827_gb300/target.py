"""A decoding cycle whose target is a transformer with a paged key/value cache.

The driver in cycles.py reads target logits from tables; here they come from a
forward pass over the pruned tree, the way a user of the library runs it: pages and
slots from the requests' lengths (cache_reserve), per layer the norms and rotation of
queries and keys with the store into the cache (qk_norm_rope) and the attention of
the drafted tree over the cache (tree_attend), verification, the log probabilities of
what was emitted (token_logprobs), and the accepted path's lines moved into place
(cache_commit).  The model is a small decoder with random weights; its projections
and products are plain torch.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import cycles, rheo


@dataclass(frozen=True)
class Shape:
    vocab: int
    layers: int = 2
    hidden: int = 128
    q_heads: int = 4
    kv_heads: int = 2
    head_dim: int = 64
    positions: int = 4096
    rot: int = 64
    eps: float = 1e-6
    dtype: str = "bf16"


class Target:
    """Weights of a decoder with RMS norms, grouped query heads with per-head norms, and a gated MLP."""

    def __init__(self, shape: Shape, seed: int = 0, device="cuda"):
        self.shape = s = shape
        dt = rheo._dtype_of(s.dtype)[1]
        g = torch.Generator(device="cpu").manual_seed(seed)

        def w(*dims, scale=None):
            x = torch.randn(dims, generator=g) * (dims[-1] ** -0.5 if scale is None else scale)
            return x.to(device=device, dtype=dt)

        heads = (s.q_heads + 2 * s.kv_heads) * s.head_dim
        self.embed = w(s.vocab, s.hidden, scale=1.0)
        self.layers = [dict(qkv=w(heads, s.hidden), out=w(s.hidden, s.q_heads * s.head_dim), up=w(4 * s.hidden, s.hidden),
                            down=w(s.hidden, 2 * s.hidden), q_norm=1 + w(s.head_dim, scale=0.1),
                            k_norm=1 + w(s.head_dim, scale=0.1)) for _ in range(s.layers)]
        self.head = w(s.vocab, s.hidden, scale=3.0 * s.hidden ** -0.5)
        at = torch.arange(s.positions, dtype=torch.float64)[:, None]
        turn = at * 10000.0 ** (-torch.arange(0, s.rot, 2, dtype=torch.float64) / s.rot)
        self.cos_sin = torch.cat([turn.cos(), turn.sin()], 1).float().to(device)

    def norm(self, x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + self.shape.eps)).to(x.dtype)


class Cached:
    """A target with its cache for `batch` requests of up to `most` tokens, `tokens` new ones a call.  With `share`,
    another one of the same sizes, it works on that one's pages: a prompt's calls and a tree's have different `tokens`."""

    def __init__(self, model: Target, batch: int, tokens: int, most: int, page_size: int = 16, share: Cached = None,
                 device="cuda"):
        s = model.shape
        width = -(-most // page_size)
        self.model = model
        self.cfg = rheo.CacheConfig(batch=batch, tokens=tokens, pages=batch * width,
                                    page_size=page_size, max_pages=width, q_heads=s.q_heads, kv_heads=s.kv_heads,
                                    head_dim=s.head_dim, dtype=s.dtype)
        if share is None:
            self.key, self.value = rheo.make_cache(self.cfg, s.layers, device)
            self.pages = rheo.Pages(self.cfg, device)
            self.ctx_len = torch.zeros(batch, dtype=torch.int32, device=device)
        else:
            self.key, self.value, self.pages, self.ctx_len = share.key, share.value, share.pages, share.ctx_len
        self.next_len = torch.zeros_like(self.ctx_len)
        self.plan, self.ws = rheo.CachePlan(self.cfg, device), rheo.CacheWorkspace(self.cfg, device)
        self.out = torch.empty((batch, tokens, s.q_heads, s.head_dim), dtype=self.cfg.torch_dtype, device=device)

    def forward(self, token: torch.Tensor, new_len=None, depth=None, mask=None) -> torch.Tensor:
        """Logits [B, T, V] of the new tokens (int, [B, T]), whose keys and values enter the cache behind ctx_len."""
        m, s, c, ws = self.model, self.model.shape, self.cfg, self.ws
        B, T, Hq, H, D = c.batch, c.tokens, s.q_heads, s.kv_heads, s.head_dim
        rheo.cache_reserve(c, self.ctx_len, self.pages, self.plan, ws, new_len=new_len, depth=depth)
        x = m.embed[token.clamp(min=0).long()]
        for i, w in enumerate(m.layers):
            qkv = m.norm(x) @ w["qkv"].T
            q, k, v = (qkv[..., a * D:b * D].unflatten(2, (b - a, D))
                       for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
            rheo.qk_norm_rope(c, q, k, v, w["q_norm"], w["k_norm"], m.cos_sin, self.plan, self.key[i], self.value[i], q, ws,
                              eps=s.eps)
            rheo.tree_attend(c, q, self.key[i], self.value[i], self.pages, self.ctx_len, self.out, ws, new_len=new_len,
                             mask=mask)
            x = x + self.out.flatten(2) @ w["out"].T
            gate, up = (m.norm(x) @ w["up"].T).chunk(2, -1)
            x = x + (torch.nn.functional.silu(gate.float()).to(x.dtype) * up) @ w["down"].T
        return m.norm(x) @ m.head.T

    def commit(self, accepted_len: torch.Tensor, accepted_nodes: torch.Tensor) -> None:
        """Keep the root and the accepted path of the last forward."""
        rheo.cache_commit(self.cfg, self.key, self.value, self.pages, self.ctx_len, accepted_len, accepted_nodes,
                          self.next_len, self.ws)
        self.ctx_len, self.next_len = self.next_len, self.ctx_len


@dataclass
class Emitted:
    tokens: torch.Tensor      # [B, cycles * (D + 1)] in order of emission, -1 behind them
    logprobs: torch.Tensor    # their log probabilities under the target at temperature T
    entropy: torch.Tensor     # entropy of the distribution that each came from
    count: torch.Tensor       # [B]
    accepted: torch.Tensor    # [B, cycles]


def decode(cfg: rheo.Config, draft: cycles.KGramLM, target: Target, prompt: torch.Tensor, temperature: torch.Tensor,
           seed: torch.Tensor, n_cycles: int, top: int = 0, page_size: int = 16) -> Emitted:
    """`n_cycles` decoding cycles behind prompts [B, L] (L > draft.k), the draft a k-gram table."""
    B, D, N, V, k, L = cfg.batch, cfg.depth, cfg.budget, cfg.vocab, draft.k, prompt.shape[1]
    dev, i32 = prompt.device, torch.int32
    most = L + n_cycles * (D + 1) + N + 1
    net = Cached(target, B, N + 1, most, page_size, device=dev)
    # the prompt but its last token, which is the first tree's root
    if L > 1:
        first = Cached(target, B, L - 1, most, page_size, net, dev)
        first.forward(prompt[:, :L - 1].to(i32))
        if rheo.scratch_status(first.ws):
            raise rheo.RheoError("device status set by the prompt")
        net.ctx_len.fill_(L - 1)
    tree, pr, out, ws = rheo.Tree(cfg, dev), rheo.Pruned(cfg, dev), rheo.VerifyOut(cfg, row_lse=False, device=dev), \
        rheo.Workspace(cfg, dev)
    attn = rheo.TreeAttn(cfg, dev)
    lcfg = rheo.LogprobConfig(rows=B * (D + 1), vocab=V, top=top, dtype=cfg.dtype, rows_per_temperature=D + 1)
    lp, lws = rheo.Logprobs(lcfg, dev), rheo.LogprobWorkspace(lcfg, dev)
    T = temperature.float().to(dev)
    width = n_cycles * (D + 1)
    got = Emitted(torch.full((B, width + D + 1), -1, dtype=torch.int64, device=dev),
                  torch.zeros((B, width + D + 1), device=dev), torch.zeros((B, width + D + 1), device=dev),
                  torch.zeros(B, dtype=torch.int64, device=dev), torch.zeros((B, n_cycles), dtype=i32, device=dev))
    window, root = prompt[:, L - k:].long(), prompt[:, -1].long()
    place = torch.arange(D + 1, device=dev)[None, :]
    base = torch.arange(B, device=dev)[:, None] * (N + 1)
    for cycle in range(n_cycles):
        offset = torch.full((B,), cycle, dtype=torch.int64, device=dev)
        for d in range(1, D + 1):
            if d == 1:
                ctx = window[:, None, :]
            else:
                path, length = cycles._paths(tree.token, tree.parent, tree.frontier.long(), d - 1)
                ctx = cycles._contexts(window, path, length, k)
            rheo.expand(cfg, d, draft.rows(ctx).to(cfg.torch_dtype).contiguous(), T, seed, offset, tree, ws)
        rheo.prune(cfg, tree, pr, ws)
        rheo.tree_attention(cfg, pr, attn, ws)
        token = torch.cat([root[:, None].to(i32), pr.token[:, 1:]], 1)
        logits = net.forward(token, depth=attn.position, mask=attn.mask).to(cfg.torch_dtype)
        rheo.verify(cfg, logits, T, seed, offset, tree, pr, out, ws)
        net.commit(out.accepted_len, out.accepted_nodes)
        # the emitted tokens and the nodes whose rows they came from: the root, then the path
        a = out.accepted_len.long()[:, None]
        toks = torch.cat([out.accepted_tokens.long(), torch.full((B, 1), -1, dtype=torch.int64, device=dev)], 1)
        toks = toks.scatter(1, a, out.bonus_token.long()[:, None])
        rows = torch.cat([torch.zeros((B, 1), dtype=torch.int64, device=dev), out.accepted_nodes.long()], 1)
        rows = torch.where(place <= a, base + rows, -1)
        rheo.token_logprobs(lcfg, logits, toks.reshape(-1).to(i32), lp, lws, temperature=T, rows=rows.reshape(-1).to(i32))
        at = got.count[:, None] + place
        got.tokens.scatter_(1, at, toks)
        got.logprobs.scatter_(1, at, lp.logprob.reshape(B, D + 1))
        got.entropy.scatter_(1, at, lp.entropy.reshape(B, D + 1))
        got.count += a[:, 0] + 1
        got.accepted[:, cycle] = out.accepted_len
        window = torch.gather(torch.cat([window, toks], 1), 1, a + 1 + torch.arange(k, device=dev)[None, :])
        root = out.bonus_token.long()
    if rheo.status(cfg, ws) or rheo.scratch_status(net.ws) or rheo.scratch_status(lws):
        raise rheo.RheoError("device status set during the cycles")
    got.tokens, got.logprobs, got.entropy = (x[:, :width] for x in (got.tokens, got.logprobs, got.entropy))
    return got


def dense_logits(target: Target, tokens: torch.Tensor) -> torch.Tensor:
    """Logits [L, V] of one sequence [L] without a cache, in 64 bits: what the cached passes have to agree with."""
    s, L = target.shape, tokens.numel()
    f = lambda w: w.double()  # noqa: E731

    def norm(x):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + s.eps)

    def turn(x):  # [L, heads, D]
        r = s.rot // 2
        c, sn = (target.cos_sin[:L, a:b].double()[:, None] for a, b in ((0, r), (r, 2 * r)))
        x0, x1, rest = x[..., :r], x[..., r:2 * r], x[..., 2 * r:]
        return torch.cat([x0 * c - x1 * sn, x1 * c + x0 * sn, rest], -1)

    x = f(target.embed[tokens.long()])
    G = s.q_heads // s.kv_heads
    for w in target.layers:
        q, k, v = (norm(x) @ f(w["qkv"]).T).split([s.q_heads * s.head_dim] + [s.kv_heads * s.head_dim] * 2, -1)
        q, k, v = (y.reshape(L, -1, s.head_dim) for y in (q, k, v))
        q, k = turn(norm(q) * f(w["q_norm"])), turn(norm(k) * f(w["k_norm"]))
        k, v = (y.repeat_interleave(G, 1) for y in (k, v))
        sc = torch.einsum("qhd,khd->hqk", q, k) * s.head_dim ** -0.5
        sc = sc.masked_fill(torch.ones((L, L), dtype=torch.bool, device=x.device).triu(1), -torch.inf)
        x = x + torch.einsum("hqk,khd->qhd", torch.softmax(sc, -1), v).reshape(L, -1) @ f(w["out"]).T
        gate, up = (norm(x) @ f(w["up"]).T).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ f(w["down"]).T
    return norm(x) @ f(target.head).T
