"""Cases of the paged key/value cache operators and of the token log probabilities.

Five operators that a target forward over a pruned draft tree needs around the
tree's expansion and verification:

  reserve    block tables, slots and positions of the new tokens from the requests' lengths
  rope       per-head RMS norms of queries and keys, the position rotation, and the store into the cache
  attend     attention of the new tokens (a drafted tree, a chain or one token) over the paged cache
  commit     the accepted path's keys and values moved to consecutive positions
  logprobs   log probabilities of given tokens, with rank, entropy and top alternatives

`run` computes each in elementary torch operations (own = False) or through the
package's entry points (own = True).  Lengths come from the case alone (an even
spread, in an order drawn from the seed), so the work of a case does not depend
on the seed.
"""
import math
import random

import numpy as np
import torch

own = False

NEG_INF = float("-inf")


# ----------------------------------------------------------------------------- cases

def _attend(name, **kw):
    c = dict(name=name, op="attend", dtype="bf16", batch=1, tokens=1, ctx_min=0, ctx_max=0, page=16, q_heads=32,
             kv_heads=8, head_dim=128, tree=True, ragged=False)
    c.update(kw)
    return c


def _rope(name, **kw):
    c = dict(name=name, op="rope", dtype="bf16", batch=1, tokens=1, ctx_min=0, ctx_max=0, page=16, q_heads=32,
             kv_heads=8, head_dim=128, rot=128, interleaved=False, norm=True, ragged=False)
    c.update(kw)
    return c


def listed():
    return [
        # plain decoding beside the trees: one token a request, contexts of every length
        _attend("attend_decode_b32", batch=32, tokens=1, ctx_min=37, ctx_max=16201, page=16, tree=False),
        # one request of a 60-node tree (the llama8b workload's budget): latency counts
        _attend("attend_tree_b1", batch=1, tokens=61, ctx_min=1911, ctx_max=1911, page=64),
        # the serving mix: 64 requests, 60-node trees, ragged contexts up to 8 thousand tokens
        _attend("attend_tree_b64", batch=64, tokens=61, ctx_min=219, ctx_max=8101, page=32),
        # a small model in fp32 (the tiny workload's budget of 16), a short cache, trees cut short
        _attend("attend_tree_f32", dtype="f32", batch=4, tokens=17, ctx_min=5, ctx_max=733, q_heads=8, kv_heads=4,
                head_dim=64, ragged=True),
        # the tiny workload's forward: fp32, half of each head rotated, pairs of neighbours
        _rope("rope_f32_small", dtype="f32", batch=3, tokens=17, ctx_min=5, ctx_max=733, q_heads=8, kv_heads=4,
              head_dim=64, rot=32, interleaved=True, ragged=True),
        # the stress workload's trees (256 requests, 128 nodes), one layer of the forward
        _rope("rope_stress", batch=256, tokens=129, ctx_min=100, ctx_max=1100, page=64),
        # one request starts its next cycle
        dict(name="reserve_b1", op="reserve", batch=1, tokens=61, ctx_min=1911, ctx_max=1911, page=16, grow=61),
        # 256 requests of long ragged contexts; some grow by a page or many, some end, some lack nothing
        dict(name="reserve_b256", op="reserve", batch=256, tokens=129, ctx_min=1, ctx_max=32003, page=16, grow=700),
        # one request's accepted path in a 32-layer cache
        dict(name="commit_b1", op="commit", dtype="bf16", batch=1, tokens=61, ctx_min=701, ctx_max=701, page=16,
             layers=32, kv_heads=8, head_dim=128, depth=6),
        # 64 requests' accepted paths
        dict(name="commit_b64", op="commit", dtype="bf16", batch=64, tokens=61, ctx_min=31, ctx_max=303, page=32,
             layers=16, kv_heads=8, head_dim=128, depth=6),
        # one row of the tiny workload
        dict(name="logprobs_tiny", op="logprobs", dtype="f32", requests=1, nodes=17, rows=4, vocab=1024, top=5,
             tempered=False, masked=0.0),
        # the emitted path of every request of the qwen3_batch workload: 16 x (8 + 1) rows of its target logits
        dict(name="logprobs_qwen3_batch", op="logprobs", dtype="bf16", requests=16, nodes=49, rows=9, vocab=151936,
             top=20, tempered=True, masked=0.0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rope", "reserve", "commit", "logprobs", "logprobs"])
    if op in ("attend", "rope"):
        f32 = rng.random() < (0.2 if op == "attend" else 0.4)
        kv_heads = rng.choice([1, 2, 4, 8] if f32 else [1, 2, 4, 8, 8, 16, 40])
        group = rng.choice([1, 2, 4] if f32 else [1, 2, 4, 4, 5, 8]) if kv_heads <= 8 else 1
        D = rng.choice([64, 128, 128])
        B = _log(rng, 1, 16 if f32 else 64)
        T = rng.choice([1, 1, 2, 17, 49, 61, rng.randint(3, 129), _log(rng, 1, 300)])
        page = rng.choice([16, 32, 64, 128])
        if op == "attend":
            # no more than the largest listed case reads (tokens x heads) and multiplies
            top = 64 * 4160 * 8 * 128 // (4 if f32 else 1)
            most = max(1, min(32768, top // (B * kv_heads * D), 64 * 4160 * 61 * 32 * 128 //
                              ((32 if f32 else 1) * B * T * kv_heads * group * D)))
            hi = _log(rng, 1, most)
            lo = rng.choice([0, hi, rng.randint(0, hi)])
            return dict(op="attend", dtype="f32" if f32 else "bf16", batch=B, tokens=T, ctx_min=lo, ctx_max=hi,
                        page=page, q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=D, tree=rng.random() < 0.7,
                        ragged=rng.random() < 0.3)
        hi = _log(rng, 1, 2000)
        rot = rng.choice([D, D, D // 2, 24])
        return dict(op="rope", dtype="f32" if f32 else "bf16", batch=B, tokens=T, ctx_min=rng.randint(0, hi),
                    ctx_max=hi, page=page, q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=D, rot=rot,
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.8, ragged=rng.random() < 0.3)
    if op == "reserve":
        hi = _log(rng, 1, 30000)
        return dict(op="reserve", batch=_log(rng, 1, 256), tokens=_log(rng, 1, 129), ctx_min=rng.randint(0, hi),
                    ctx_max=hi, page=rng.choice([16, 32, 64, 128]), grow=_log(rng, 1, 700))
    if op == "commit":
        depth = rng.randint(1, 10)
        hi = _log(rng, 1, 300)
        return dict(op="commit", dtype=rng.choice(["bf16", "bf16", "f32"]), batch=_log(rng, 1, 48),
                    tokens=rng.randint(2 * depth + 2, 129), ctx_min=rng.randint(0, hi), ctx_max=hi,
                    page=rng.choice([16, 32, 64]), layers=rng.randint(1, 12), kv_heads=rng.choice([1, 2, 4, 8]),
                    head_dim=rng.choice([64, 128]), depth=depth)
    f32 = rng.random() < 0.4
    V = _log(rng, 300, 262144)
    rows = rng.randint(1, 11)
    requests = max(1, min(_log(rng, 1, 64), (144 if f32 else 288) * 151936 // (2 * V * rows)))
    return dict(op="logprobs", dtype="f32" if f32 else "bf16", requests=requests, nodes=rng.randint(rows, rows + 30),
                rows=rows, vocab=V, top=rng.choice([0, 1, 5, 20, 32]), tempered=rng.random() < 0.7,
                masked=rng.choice([0.0, 0.0, 0.5, 0.99]))


def _spread(case):
    """Context lengths and new tokens of the requests, in order of length."""
    B, T, lo, hi = case["batch"], case["tokens"], case["ctx_min"], case["ctx_max"]
    ctx = [lo + (hi - lo) * b // max(B - 1, 1) for b in range(B)]
    if B == 1:
        ctx = [hi]
    new = [1 + (7 * b + 3) % T if case.get("ragged") else T for b in range(B)]
    return ctx, new


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "attend":
        ctx, new = _spread(case)
        s, H, D, T, B = _size(case), case["kv_heads"], case["head_dim"], case["tokens"], case["batch"]
        kv = sum(c + n for c, n in zip(ctx, new)) * H * D * 2 * s
        q = sum(new) * case["q_heads"] * D * s
        out = B * T * case["q_heads"] * (D * s + 4)
        mask = sum(n * n for n in new) if case["tree"] else 0
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
        return {"bytes": kv + q + out + mask, "flops": 4 * D * case["q_heads"] * pairs}
    if op == "rope":
        _, new = _spread(case)
        s, D, n = _size(case), case["head_dim"], sum(new)
        heads = case["q_heads"] + 2 * case["kv_heads"]
        return {"bytes": 2 * n * heads * D * s + n * 12, "flops": 8 * n * (heads - case["kv_heads"]) * D}
    if op == "reserve":
        ctx, new = _spread(case)
        B, T = case["batch"], case["tokens"]
        pages = sum(-(-(c + n) // case["page"]) for c, n in zip(ctx, new))
        return {"bytes": 8 * pages + B * T * 16 + 12 * B, "flops": 0}
    if op == "commit":
        moved = sum(_accepted(case, b) for b in range(case["batch"]))
        return {"bytes": moved * case["layers"] * case["kv_heads"] * case["head_dim"] * 4 * _size(case), "flops": 0}
    n = case["requests"] * case["rows"]
    return {"bytes": n * case["vocab"] * _size(case) + n * (16 + 8 * case["top"]), "flops": 4 * n * case["vocab"]}


def _accepted(case, b):
    """Accepted draft tokens of the b-th request: 0..depth, three on average where the tree is that deep."""
    return min(case["depth"], (5 * b + 4) % 7)


# ----------------------------------------------------------------------------- inputs

class _State:
    pass


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, seed):
    ctx, new = _spread(case)
    order = list(range(len(ctx)))
    random.Random(seed).shuffle(order)
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor([ctx[i] for i in order], **i32), torch.tensor([new[i] for i in order], **i32), order


def _trees(g, B, T):
    """Random drafted trees of T nodes: ancestor masks [B, T, T] (uint8) and depths [B, T] (int32)."""
    at = torch.arange(T, device="cuda")
    up = (at / 8).floor() if T > 1 else at.float()  # eight children a node, shallow trees as a pruned one
    back = (torch.rand((B, T), generator=g, device="cuda") * (at - up)).floor().long()
    parent = (up.long() + back).clamp(max=(at - 1).clamp(min=0))
    a = torch.zeros((B, T, T), device="cuda")
    a.scatter_(2, parent[:, :, None], 1.0)
    a[:, 0] = 0
    a += torch.eye(T, device="cuda")
    hops = 1
    while hops < T:
        a = (torch.bmm(a, a) > 0).float()
        hops *= 2
    return a.to(torch.uint8), (a.sum(2) - 1).to(torch.int32)


def _pages_of(case, g, lens, slack=3):
    """A pool whose pages are handed out in random order; the table of `lens` tokens a request."""
    P, B = case["page"], case["batch"]
    need = (lens.long() + P - 1) // P
    width = int(need.max()) + slack
    total = int(need.sum()) + slack
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(need, 0) - need
    j = torch.arange(width, device="cuda")[None, :]
    held = j < need[:, None]
    table = torch.where(held, order[(first[:, None] + j).clamp(max=total - 1)], torch.zeros_like(j, dtype=torch.int32))
    return table.to(torch.int32).contiguous(), need.to(torch.int32), total, width


def _slots(table, pos, P):
    return torch.gather(table.long(), 1, (pos // P).clamp(max=table.shape[1] - 1)) * P + pos % P


def prepare(case, seed):
    s, g = _State(), _gen(seed)
    s.case, s.op = dict(case), case["op"]
    if s.op == "attend":
        _prepare_attend(s, case, seed, g)
    elif s.op == "rope":
        _prepare_rope(s, case, seed, g)
    elif s.op == "reserve":
        _prepare_reserve(s, case, seed, g)
    elif s.op == "commit":
        _prepare_commit(s, case, seed, g)
    else:
        _prepare_logprobs(s, case, seed, g)
    if own:
        _handles(s, case)
    return s


def _prepare_attend(s, case, seed, g):
    B, T, H, Hq, D, dt = case["batch"], case["tokens"], case["kv_heads"], case["q_heads"], case["head_dim"], _dtype(case)
    s.ctx, s.new, _ = _lengths(case, seed)
    if not case["ragged"]:
        s.new = None
    lens = s.ctx + (s.new if s.new is not None else T)
    s.table, _, s.pages, s.width = _pages_of(case, g, lens)
    s.longest = int(lens.max())
    s.mask = _trees(g, B, T)[0] if case["tree"] else None
    # normed and rotated queries and keys: scores of a few units, a common direction that some heads attend to
    shape = (s.pages, H, case["page"], D)
    s.key = torch.randn(shape, generator=g, device="cuda", dtype=dt)
    s.key += 0.5 * torch.randn((1, H, 1, D), generator=g, device="cuda", dtype=dt)
    s.value = torch.randn(shape, generator=g, device="cuda", dtype=dt)
    s.q = 1.5 * torch.randn((B, T, Hq, D), generator=g, device="cuda", dtype=dt)
    s.scale = 1.0 / math.sqrt(D)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty((B, T, Hq), dtype=torch.float32, device="cuda")


def _prepare_rope(s, case, seed, g):
    B, T, H, Hq, D, dt = case["batch"], case["tokens"], case["kv_heads"], case["q_heads"], case["head_dim"], _dtype(case)
    P, rot = case["page"], case["rot"]
    s.ctx, s.new, _ = _lengths(case, seed)
    s.table, _, s.pages, s.width = _pages_of(case, g, s.ctx + s.new, slack=1)
    depth = _trees(g, B, T)[1].long()
    t = torch.arange(T, device="cuda")[None, :]
    live = t < s.new[:, None]
    s.slot = torch.where(live, _slots(s.table, s.ctx.long()[:, None] + t, P), torch.full_like(t, -1))
    s.position = torch.where(live, s.ctx.long()[:, None] + depth, torch.full_like(t, -1)).to(torch.int32)
    # one product gives queries, keys and values side by side
    s.qkv = torch.randn((B, T, (Hq + 2 * H) * D), generator=g, device="cuda", dtype=dt)
    s.q = s.qkv[:, :, : Hq * D].unflatten(2, (Hq, D))
    s.k = s.qkv[:, :, Hq * D: (Hq + H) * D].unflatten(2, (H, D))
    s.v = s.qkv[:, :, (Hq + H) * D:].unflatten(2, (H, D))
    s.q_weight = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) if case["norm"] else None
    s.k_weight = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) if case["norm"] else None
    s.eps = 1e-6
    at = torch.arange(int(s.position.max()) + 1, device="cuda", dtype=torch.float64)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    ang = at[:, None] * inv[None, :]
    s.cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float()
    s.key = torch.zeros((s.pages, H, P, D), device="cuda", dtype=dt)
    s.value = torch.zeros_like(s.key)
    s.q_out = torch.empty((B, T, Hq, D), device="cuda", dtype=dt)


def _prepare_reserve(s, case, seed, g):
    B, T, P = case["batch"], case["tokens"], case["page"]
    s.ctx, s.new, order = _lengths(case, seed)
    if case.get("batch") > 3:  # some requests have ended: their pages go back
        ended = torch.tensor([b % 16 == 5 for b in order], device="cuda")
        held = s.ctx.clone()
        s.ctx = torch.where(ended, torch.zeros_like(s.ctx), s.ctx)
        s.new = torch.where(ended, torch.zeros_like(s.new), s.new)
    else:
        held = s.ctx.clone()
    # what is held from before: fewer pages than the lengths ask for by up to `grow` tokens
    back = torch.randint(0, case["grow"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    owned = (torch.clamp(held - back + T, min=0).long() + P - 1) // P
    # a pool and a table that would hold every request in full, and a little more
    full = [-(-(c + T) // P) for c in _spread(case)[0]]
    s.width, s.pages = max(full) + 1, sum(full) + 7
    order = torch.randperm(s.pages, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(owned, 0) - owned
    j = torch.arange(s.width, device="cuda")[None, :]
    s.table = torch.where(j < owned[:, None], order[(first[:, None] + j).clamp(max=s.pages - 1)],
                          torch.full_like(j, -1, dtype=torch.int32)).to(torch.int32).contiguous()
    s.n_pages = owned.to(torch.int32)
    s.n_free = (s.pages - owned.sum()).to(torch.int32).reshape(1)
    at = torch.arange(s.pages, device="cuda")
    s.free = torch.where(at < s.n_free, order.flip(0)[at], torch.full_like(at, -1, dtype=torch.int32)).to(torch.int32)
    s.depth = _trees(g, B, T)[1]


def _prepare_commit(s, case, seed, g):
    B, T, P, D, depth = case["batch"], case["tokens"], case["page"], case["head_dim"], case["depth"]
    s.ctx, _, order = _lengths(case, seed)
    s.table, _, s.pages, s.width = _pages_of(case, g, s.ctx + T)
    shape = (case["layers"], s.pages, case["kv_heads"], P, D)
    s.key = torch.randn(shape, generator=g, device="cuda", dtype=_dtype(case))
    s.value = torch.randn(shape, generator=g, device="cuda", dtype=_dtype(case))
    s.accepted_len = torch.tensor([_accepted(case, b) for b in order], dtype=torch.int32, device="cuda")
    # ascending nodes: the first child's line for a while, then nodes past every place that is written
    r, rows = random.Random(seed + 1), []
    for b in range(B):
        a, path = int(_accepted(case, order[b])), []
        stay = r.randint(0, a)
        later = sorted(r.sample(range(depth + 1, T), depth))
        for k in range(depth):
            path.append(-1 if k >= a else k + 1 if k < stay else later[k])
        rows.append(path)
    s.accepted_nodes = torch.tensor(rows, dtype=torch.int32, device="cuda")
    s.next_len = torch.empty_like(s.ctx)


def _prepare_logprobs(s, case, seed, g):
    B, N, R, V, dt = case["requests"], case["nodes"], case["rows"], case["vocab"], _dtype(case)
    # Zipf-shaped logits, as a language model's: -1.2 ln(rank) at a random rank, and noise
    x = torch.rand((B * N, V), generator=g, device="cuda")
    x = -1.2 * torch.log(1 + x * V)
    x += 0.5 * torch.randn((B * N, V), generator=g, device="cuda")
    if case["masked"]:
        x = torch.where(torch.rand((B * N, V), generator=g, device="cuda") < case["masked"], NEG_INF, x)
        x[:, V // 3] = 1.0
    s.logits = x.to(dt)
    # the emitted path: the root's row, then accepted nodes' rows; a path that ends early leaves rows out
    r = torch.randint(0, N, (B, R), generator=g, device="cuda")
    r = r + torch.arange(B, device="cuda")[:, None] * N
    if R > 2:
        gone = torch.rand((B, 1), generator=g, device="cuda") < 0.2
        r[:, -1:] = torch.where(gone, torch.full_like(gone, -1, dtype=r.dtype), r[:, -1:])
    s.rows = r.reshape(-1).to(torch.int32)
    # given tokens: likely ones mostly, any now and then
    picked = s.logits[s.rows.clamp(min=0).long()].float()
    noise = -torch.log(-torch.log(torch.rand(picked.shape, generator=g, device="cuda").clamp(1e-20, 1 - 1e-7)))
    s.tokens = (picked + noise).argmax(1).to(torch.int32)
    s.temperature = None
    if case["tempered"]:
        s.temperature = 0.5 + torch.rand(B, generator=g, device="cuda")


def _handles(s, case):
    """What a user of the package holds beside the tensors: configurations, workspaces, output buffers."""
    from paper_2609_21827_gb300 import rheo

    s.rheo = rheo
    if s.op == "logprobs":
        n = case["requests"] * case["rows"]
        s.cfg = rheo.LogprobConfig(rows=n, vocab=case["vocab"], top=case["top"], dtype=case["dtype"],
                                   rows_per_temperature=case["rows"])
        s.out, s.ws = rheo.Logprobs(s.cfg), rheo.LogprobWorkspace(s.cfg)
        return
    s.cfg = rheo.CacheConfig(batch=case["batch"], tokens=case["tokens"], pages=s.pages, page_size=case["page"],
                             max_pages=s.width, q_heads=case.get("q_heads", case.get("kv_heads", 1)),
                             kv_heads=case.get("kv_heads", 1), head_dim=case.get("head_dim", 64),
                             dtype=case.get("dtype", "bf16"))
    s.ws = rheo.CacheWorkspace(s.cfg)
    if s.op in ("attend", "commit"):
        s.held = rheo.Pages(s.cfg, block_table=s.table)
    elif s.op == "reserve":
        s.held = rheo.Pages(s.cfg, block_table=s.table, n_pages=s.n_pages, free_list=s.free, n_free=s.n_free)
        s.after = rheo.Pages(s.cfg)
        s.plan = rheo.CachePlan(s.cfg)
    else:
        s.plan = rheo.CachePlan(s.cfg, slot=s.slot, position=s.position)


# ----------------------------------------------------------------------------- one pass

def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s.op](s)


def _own_attend(s):
    s.rheo.tree_attend(s.cfg, s.q, s.key, s.value, s.held, s.ctx, s.out, s.ws, new_len=s.new, mask=s.mask, lse=s.lse,
                       scale=s.scale)
    return {"out": s.out, "lse": s.lse}


def _own_rope(s):
    s.rheo.qk_norm_rope(s.cfg, s.q, s.k, s.v, s.q_weight, s.k_weight, s.cos_sin, s.plan, s.key, s.value, s.q_out, s.ws,
                        eps=s.eps, interleaved=s.case["interleaved"])
    return {"q": s.q_out, "key": s.key, "value": s.value}


def _own_reserve(s):
    s.rheo.cache_reserve(s.cfg, s.ctx, s.held, s.plan, s.ws, new_len=s.new, depth=s.depth, out=s.after)
    a = s.after
    return {"table": a.block_table, "n_pages": a.n_pages, "free": a.free_list, "n_free": a.n_free,
            "slot": s.plan.slot, "position": s.plan.position}


def _own_commit(s):
    s.rheo.cache_commit(s.cfg, s.key, s.value, s.held, s.ctx, s.accepted_len, s.accepted_nodes, s.next_len, s.ws)
    return {"key": s.key, "value": s.value, "next_len": s.next_len}


def _own_logprobs(s):
    s.rheo.token_logprobs(s.cfg, s.logits, s.tokens, s.out, s.ws, temperature=s.temperature, rows=s.rows)
    o = s.out
    got = {"logprob": o.logprob, "rank": o.rank, "entropy": o.entropy}
    if s.case["top"]:
        got["top_ids"], got["top_logprobs"] = o.top_ids, o.top_logprobs
    return got


def _visible(ctx, new, mask, T, L):
    """[B, T, L]: whether new token t sees position l of its request."""
    dev = ctx.device
    l, t = torch.arange(L, device=dev)[None, None, :], torch.arange(T, device=dev)[None, :, None]
    j = l - ctx.long()[:, None, None]
    n = torch.full_like(ctx, T) if new is None else new
    if mask is None:
        among = j <= t
    else:
        among = torch.gather(mask, 2, j.clamp(0, T - 1).expand(-1, T, -1)) != 0
    return ((j < 0) | (among & (j < n.long()[:, None, None]))) & (t < n.long()[:, None, None])


def _plain_attend(s):
    c = s.case
    P, L, H, G, D, B, T = c["page"], s.longest, c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["batch"], \
        c["tokens"]
    at = torch.arange(L, device="cuda")
    page = s.table[:, at // P].long()                              # [B, L]
    n = s.ctx + (T if s.new is None else s.new)
    held = (at[None, :] < n[:, None])[:, None, :, None]
    k = s.key[page, :, at % P].permute(0, 2, 1, 3).float()         # [B, H, L, D]
    v = torch.where(held, s.value[page, :, at % P].permute(0, 2, 1, 3).float(), 0.0)
    q = s.q.float().reshape(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    x = torch.matmul(q, k.transpose(2, 3)) * s.scale               # [B, H, T*G, L]
    seen = _visible(s.ctx, s.new, s.mask, T, L)
    x = x.reshape(B, H, T, G, L)
    x = torch.where(seen[:, None, :, None, :], x, NEG_INF)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == NEG_INF, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, H, T * G, L), v).reshape(B, H, T, G, D)
    o = torch.where(z > 0, o / z, torch.zeros_like(o))
    lse = (m + torch.log(z)).squeeze(-1)
    return {"out": o.permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(s.q.dtype),
            "lse": lse.permute(0, 2, 1, 3).reshape(B, T, H * G)}


def _rotate(x, cos, sin, rot, interleaved):
    """x [B, T, heads, D] float; cos, sin [B, T, 1, rot / 2]."""
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., : rot // 2], r[..., rot // 2:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1)


def _plain_rope(s):
    c = s.case
    rot, dt = c["rot"], s.q.dtype
    live = s.slot >= 0
    cs = s.cos_sin[s.position.clamp(min=0).long()][:, :, None, :]
    cos, sin = cs[..., : rot // 2], cs[..., rot // 2:]

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s.eps) * w.float()
        return _rotate(x, cos, sin, rot, c["interleaved"]).to(dt)

    q = torch.where(live[:, :, None, None], one(s.q, s.q_weight), torch.zeros((), dtype=dt, device="cuda"))
    # tokens without a slot store the request's first token once more
    at = torch.where(live, s.slot, s.slot[:, :1])
    k, v = (torch.where(live[:, :, None, None], x, x[:, :1]) for x in (one(s.k, s.k_weight), s.v))
    s.key[at // c["page"], :, at % c["page"]] = k
    s.value[at // c["page"], :, at % c["page"]] = v
    return {"q": q, "key": s.key, "value": s.value}


def _plain_reserve(s):
    c = s.case
    P, T = c["page"], c["tokens"]
    own_, free0, dev = s.n_pages.long(), s.n_free.long(), "cuda"
    need = (s.ctx.long() + s.new.long() + P - 1) // P
    fits = need <= s.width
    back = torch.where(fits, (own_ - need).clamp(min=0), 0)
    want = torch.where(fits, (need - own_).clamp(min=0), 0)
    j = torch.arange(s.width, device=dev)[None, :]
    # released pages go on the stack in order of request, then of place
    keep = own_ - back
    dest = free0 + (torch.cumsum(back, 0) - back)[:, None] + j - keep[:, None]
    dest = torch.where((j >= keep[:, None]) & (j < own_[:, None]), dest, s.pages)
    free = torch.cat([s.free, s.free.new_zeros(1)])
    free = free.scatter(0, dest.reshape(-1), s.table.reshape(-1))[: s.pages]
    have = free0 + back.sum()
    upto = torch.cumsum(want, 0)
    ok = (upto <= have) & fits
    take = torch.where(ok, want, 0)
    src = have - 1 - ((upto - want)[:, None] + j - own_[:, None])
    got = (j >= own_[:, None]) & (j < (own_ + take)[:, None])
    table = torch.where(got, free[src.clamp(0, s.pages - 1)], s.table)
    t = torch.arange(T, device=dev)[None, :]
    live = (t < s.new[:, None]) & ok[:, None]
    pos = s.ctx.long()[:, None] + t
    slot = torch.where(live, _slots(table, pos, P), torch.full_like(pos, -1))
    where = torch.where(live, s.ctx.long()[:, None] + s.depth.long(), torch.full_like(pos, -1))
    return {"table": table, "n_pages": (own_ - back + take).to(torch.int32), "free": free,
            "n_free": (have - take.sum()).to(torch.int32), "slot": slot, "position": where.to(torch.int32)}


def _plain_commit(s):
    c = s.case
    P, D = c["page"], c["depth"]
    k = torch.arange(D, device="cuda")[None, :]
    live = k < s.accepted_len[:, None]  # places past the path copy the root's line onto itself
    src = _slots(s.table, s.ctx.long()[:, None] + torch.where(live, s.accepted_nodes.long(), 0), P).reshape(-1)
    dst = _slots(s.table, s.ctx.long()[:, None] + torch.where(live, k + 1, 0), P).reshape(-1)
    for x in (s.key, s.value):
        x[:, dst // P, :, dst % P] = x[:, src // P, :, src % P]
    s.next_len = s.ctx + 1 + s.accepted_len
    return {"key": s.key, "value": s.value, "next_len": s.next_len}


def _plain_logprobs(s):
    c = s.case
    V, k, per = c["vocab"], c["top"], c["rows"]
    raw = s.logits[s.rows.clamp(min=0).long()].float() + 0.0  # no negative zero
    skip = s.rows < 0
    T = torch.ones(c["requests"], device="cuda") if s.temperature is None else s.temperature
    x = raw / T.repeat_interleave(per)[:, None]
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    lse = m + torch.log(z)
    entropy = torch.log(z) - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / z
    at = s.tokens.long()[:, None]
    l = torch.gather(raw, 1, at)
    ids = torch.arange(V, device="cuda")[None, :]
    rank = ((raw > l) | ((raw == l) & (ids < at))).sum(1)
    logprob = (torch.gather(x, 1, at) - lse).squeeze(1)
    got = {"logprob": torch.where(skip, 0.0, logprob),
           "rank": torch.where(skip, -1, rank).to(torch.int32),
           "entropy": torch.where(skip, 0.0, entropy.squeeze(1))}
    if k:
        n = min(k, V)
        bits = raw.contiguous().view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()  # whole numbers in the order of the logits
        top = torch.topk(order * (1 << 32) + (V - 1 - ids), n, dim=1).values
        top_ids = V - 1 - (top & 0xFFFFFFFF)
        lp = torch.gather(x, 1, top_ids) - lse
        none = skip[:, None] | (lp == NEG_INF)
        got["top_ids"] = torch.where(none, -1, top_ids).to(torch.int32)
        got["top_logprobs"] = torch.where(none, NEG_INF, lp)
    return got


_RUN_OWN = {"attend": _own_attend, "rope": _own_rope, "reserve": _own_reserve, "commit": _own_commit,
            "logprobs": _own_logprobs}
_RUN_PLAIN = {"attend": _plain_attend, "rope": _plain_rope, "reserve": _plain_reserve, "commit": _plain_commit,
              "logprobs": _plain_logprobs}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "rope": _exact_rope, "reserve": _exact_reserve, "commit": _exact_commit,
            "logprobs": _exact_logprobs}[case["op"]](s, case)


def _exact_attend(s, c):
    """Request by request: softmax(q k / sqrt(D)) v over the positions that a token sees."""
    B, T, H, D, P = c["batch"], c["tokens"], c["kv_heads"], c["head_dim"], c["page"]
    G = c["q_heads"] // H
    out = torch.zeros((B, T, H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H * G), NEG_INF, dtype=torch.float64, device="cuda")
    ctx = s.ctx.tolist()
    new = [T] * B if s.new is None else s.new.tolist()
    for b in range(B):
        n, L = new[b], ctx[b] + new[b]
        pages = s.table[b, : -(-L // P)].long()
        k = s.key[pages].double().transpose(0, 1).reshape(H, -1, D)[:, :L]
        v = s.value[pages].double().transpose(0, 1).reshape(H, -1, D)[:, :L]
        seen = torch.ones((n, L), dtype=torch.bool, device="cuda")
        if s.mask is not None:
            seen[:, ctx[b]:] = s.mask[b, :n, :n] != 0
        else:
            seen[:, ctx[b]:] = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        for h in range(H):
            q = s.q[b, :n, h * G:(h + 1) * G].double()                       # [n, G, D]
            x = (q.reshape(n * G, D) @ k[h].T).reshape(n, G, L) * s.scale
            x.masked_fill_(~seen[:, None, :], NEG_INF)
            w = torch.logsumexp(x, -1, keepdim=True)
            p = torch.exp(x - w).nan_to_num(0.0)
            out[b, :n, h * G:(h + 1) * G] = (p.reshape(n * G, L) @ v[h]).reshape(n, G, D)
            lse[b, :n, h * G:(h + 1) * G] = w[..., 0]
    return {"out": out, "lse": lse}


def _exact_rope(s, c):
    """Neighbours or halves as complex numbers, turned by position x 10000^(-2i / rot)."""
    rot, D = c["rot"], c["head_dim"]
    angle = s.position.clamp(min=0).double()[:, :, None] * \
        (10000.0 ** (-2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot))
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None, :]

    def one(x, w):
        x = x.double()
        if w is not None:
            x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + s.eps)
        y = x.clone()
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., a], x[..., b]) * turn
        y[..., a], y[..., b] = z.real, z.imag
        return y

    q, k = one(s.q, s.q_weight), one(s.k, s.k_weight)
    q = q * (s.slot >= 0)[:, :, None, None]
    key, value = s.key.double(), s.value.double()
    b, t = torch.nonzero(s.slot >= 0, as_tuple=True)
    page, row = s.slot[b, t] // c["page"], s.slot[b, t] % c["page"]
    key[page, :, row] = k[b, t]
    value[page, :, row] = s.v[b, t].double()
    return {"q": q, "key": key, "value": value}


def _exact_reserve(s, c):
    """The stack of free pages, played through request by request."""
    P, T = c["page"], c["tokens"]
    table, owned = s.table.tolist(), s.n_pages.tolist()
    free, top = s.free.tolist(), int(s.n_free)
    ctx, new, depth = s.ctx.tolist(), s.new.tolist(), s.depth.tolist()
    need = [-(-(a + b) // P) for a, b in zip(ctx, new)]
    for b in range(c["batch"]):
        for j in range(need[b], owned[b]):
            free[top] = table[b][j]
            top += 1
        owned[b] = min(owned[b], need[b])
    stack, dry, ok = top, False, []
    for b in range(c["batch"]):
        want = need[b] - owned[b]
        dry = dry or want > stack
        ok.append(not dry or want == 0)
        if want and not dry:
            for j in range(owned[b], need[b]):
                stack -= 1
                table[b][j] = free[stack]
            owned[b] = need[b]
    slot, position = np.full((c["batch"], T), -1, np.int64), np.full((c["batch"], T), -1, np.int32)
    for b in range(c["batch"]):
        for t in range(new[b] if ok[b] else 0):
            x = ctx[b] + t
            slot[b, t], position[b, t] = table[b][x // P] * P + x % P, ctx[b] + depth[b][t]
    return {"table": np.array(table, np.int32), "n_pages": np.array(owned, np.int32), "free": np.array(free, np.int32),
            "n_free": np.array([stack], np.int32), "slot": slot, "position": position}


def _exact_commit(s, c):
    """Each request's accepted nodes, in order, copied to the positions behind its root."""
    P = c["page"]
    key, value = s.key.clone(), s.value.clone()
    ctx, table = s.ctx.tolist(), s.table.tolist()
    for b, (n, nodes) in enumerate(zip(s.accepted_len.tolist(), s.accepted_nodes.tolist())):
        for k in range(n):
            x, y = ctx[b] + nodes[k], ctx[b] + k + 1
            for z in (key, value):
                z[:, table[b][y // P], :, y % P] = z[:, table[b][x // P], :, x % P]
    return {"key": key, "value": value, "next_len": torch.tensor([a + 1 + n for a, n in zip(ctx, s.accepted_len.tolist())],
                                                                 dtype=torch.int32)}


def _exact_logprobs(s, c):
    """log softmax and its entropy row by row; places by a stable sort."""
    R, V, k = s.rows.numel(), c["vocab"], min(c["top"], c["vocab"])
    got = {"logprob": torch.zeros(R, dtype=torch.float64), "rank": torch.full((R,), -1, dtype=torch.int32),
           "entropy": torch.zeros(R, dtype=torch.float64)}
    if k:
        got["top_ids"] = torch.full((R, k), -1, dtype=torch.int32)
        got["top_logprobs"] = torch.full((R, k), NEG_INF, dtype=torch.float64)
    T = None if s.temperature is None else s.temperature.double()
    for i, (r, t) in enumerate(zip(s.rows.tolist(), s.tokens.tolist())):
        if r < 0:
            continue
        x = s.logits[r].double()
        order = torch.sort(x, descending=True, stable=True).indices
        y = torch.log_softmax(x if T is None else x / T[i // c["rows"]], 0)
        p = y.exp()
        got["logprob"][i] = y[t]
        got["rank"][i] = int((order == t).nonzero()[0, 0])
        got["entropy"][i] = -(p * y)[p > 0].sum()
        if k:
            top = order[:k]
            fine = (y[top] > NEG_INF).cpu()
            got["top_ids"][i] = torch.where(fine, top.cpu(), -1).to(torch.int32)
            got["top_logprobs"][i] = y[top].cpu()
    return got
