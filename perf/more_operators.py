"""Cases of the operators for long contexts: attention limited to a window, and a cache held in 4 bits.

  window   attention of the new tokens over the paged cache, limited to a window and a few first tokens that stay visible
  pack     whole pages of the 16-bit cache turned into 4-bit pages, with the tables of both
  unpack   4-bit pages turned back into 16-bit ones
  packed   attention over 4-bit pages and, behind them, the 16-bit pages of the latest tokens

`run` computes each in elementary torch operations (own = False) or through the
package's entry points (own = True).  Lengths come from the case alone (an even
spread, in an order drawn from the seed), so the work of a case does not depend
on the seed.

A 4-bit page of one head is made of blocks of N = min(page, 32) tokens by D
channels; a block holds the keys' codes, the values' codes, a scale byte for each
channel of the keys (over the N tokens) and one for each token and 32 channels of
the values.  Scale byte c stands for s = (1 + (c & 7) / 8) 2^((c >> 3) - 19), the
smallest with 7 s >= the largest magnitude that it covers; a code is n + 8 with
n = x / s rounded to the nearest of -7 .. 7 (a half away from 0).
"""
import math
import random

import numpy as np
import torch

own = False

NEG_INF = float("-inf")


# ----------------------------------------------------------------------------- cases

def _attend(name, op, **kw):
    c = dict(name=name, op=op, dtype="bf16", batch=1, tokens=1, ctx_min=0, ctx_max=0, page=16, q_heads=32, kv_heads=8,
             head_dim=128, window=0, sinks=0, tree=True, ragged=False, keep=0)
    c.update(kw)
    return c


def _pages(name, op, **kw):
    c = dict(name=name, op=op, batch=1, ctx_min=0, ctx_max=0, page=64, keep=0, layers=1, kv_heads=8, head_dim=128)
    c.update(kw)
    return c


def listed():
    return [
        # a small fp32 model's windowed layer (the tiny workload's budget of 16), a short cache, trees cut short
        _attend("window_tree_f32", "window", dtype="f32", batch=4, tokens=17, ctx_min=5, ctx_max=733, q_heads=8, kv_heads=4,
                head_dim=64, window=100, sinks=3, ragged=True),
        # plain decoding in a windowed layer: one token a request, contexts of every length, four first tokens kept
        _attend("window_decode_b32", "window", batch=32, ctx_min=37, ctx_max=16201, window=1024, sinks=4, tree=False),
        # a piece of two prompts, in a windowed layer behind what is cached
        _attend("window_prompt_b2", "window", batch=2, tokens=2000, ctx_min=411, ctx_max=5003, page=64, window=1024, sinks=16,
                tree=False),
        # the serving mix: 64 requests, 60-node trees, contexts up to 8 thousand tokens
        _attend("window_tree_b64", "window", batch=64, tokens=61, ctx_min=219, ctx_max=8101, page=32, window=2048, sinks=64),
        # one request's page has filled up while it decodes, in a 32-layer cache
        _pages("pack_b1", "pack", ctx_min=64 * 2 + 9, ctx_max=64 * 2 + 9, keep=64, layers=32),
        # the prompts of 16 requests right after they were read, 128 tokens of each stay as they are
        _pages("pack_b16", "pack", batch=16, ctx_min=503, ctx_max=9001, keep=128, layers=4),
        # a few pages of a small cache
        _pages("unpack_small", "unpack", ctx_min=70, ctx_max=70, page=16, kv_heads=2, head_dim=64),
        # a shared prefix's pages on their way back into a 16-bit cache
        _pages("unpack_prefix", "unpack", batch=3, ctx_min=4099, ctx_max=12001, page=64, layers=8),
        # one request of a 60-node tree (the llama8b workload's budget): latency counts
        _attend("packed_tree_b1", "packed", tokens=61, ctx_min=1911, ctx_max=1911, page=16, keep=64),
        # plain decoding over long ragged contexts
        _attend("packed_decode_b32", "packed", batch=32, ctx_min=37, ctx_max=16201, page=64, keep=64, tree=False),
        # two drafted tokens a request in a chain, heads of 64, a wide window over longer contexts
        _attend("packed_window_b48", "packed", batch=48, tokens=3, ctx_min=1000, ctx_max=32003, page=128, q_heads=16,
                kv_heads=4, head_dim=64, window=8192, sinks=64, tree=False, keep=128),
        # the serving mix over 4-bit pages
        _attend("packed_tree_b64", "packed", batch=64, tokens=61, ctx_min=219, ctx_max=8101, page=32, keep=32),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    op = rng.choice(["window", "window", "packed", "packed", "packed", "pack", "unpack"])
    page = rng.choice([16, 32, 64, 128])
    if op in ("pack", "unpack"):
        H, D, layers = rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), rng.randint(1, 8)
        B = _log(rng, 1, 32)
        # at most 300 million elements of keys, as the largest listed case
        hi = page + _log(rng, 1, max(1, min(16000, 150_000_000 // (B * H * D * layers))))
        keep = 0 if op == "unpack" else min(hi - page, rng.choice([0, 0, 1, page, rng.randint(0, 100)]))
        return dict(op=op, batch=B, ctx_min=rng.choice([page, hi, rng.randint(page, hi)]), ctx_max=hi, page=page, keep=keep,
                    layers=layers, kv_heads=H, head_dim=D)
    f32 = op == "window" and rng.random() < 0.25
    H = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4] if f32 else [1, 2, 4, 4, 5, 8])
    D = rng.choice([64, 128, 128])
    T = rng.choice([1, 1, 2, 3, 17, 49, 61, rng.randint(4, 129), _log(rng, 1, 1000)])
    B = max(1, min(_log(rng, 1, 16 if f32 else 64), 4000 // T))
    # no more than the largest listed cases read, multiply, or hold as scores in the plain form
    hi = min(16384, 64 * 4160 * 8 * 128 // (4 if f32 else 1) // (B * H * D),
             64 * 4160 * 61 * 32 * 128 // ((32 if f32 else 1) * B * T * H * G * D), 500_000_000 // (B * T * H * G) - T)
    hi = _log(rng, 1, max(1, hi))
    lo = rng.choice([0, hi, rng.randint(0, hi)])
    limited = op == "window" or rng.random() < 0.5
    return dict(op=op, dtype="f32" if f32 else "bf16", batch=B, tokens=T, ctx_min=lo, ctx_max=hi, page=page, q_heads=H * G,
                kv_heads=H, head_dim=D, window=_log(rng, 1, 8192) if limited else 0,
                sinks=rng.choice([0, 1, 4, 64, rng.randint(0, 300)]) if limited else 0, tree=rng.random() < 0.6,
                ragged=rng.random() < 0.3, keep=rng.choice([0, 1, page, rng.randint(0, 200)]) if op == "packed" else 0)


def _spread(case):
    """Cached and new tokens of the requests, in order of length."""
    B, lo, hi = case["batch"], case["ctx_min"], case["ctx_max"]
    ctx = [lo + (hi - lo) * b // max(B - 1, 1) for b in range(B)]
    if B == 1:
        ctx = [hi]
    T = case.get("tokens", 0)
    return ctx, [1 + (7 * b + 3) % T if case.get("ragged") else T for b in range(B)]


def _whole(case, ctx):
    """Pages that are, or are to be, in 4 bits."""
    return max(0, (ctx - case["keep"]) // case["page"])


def _page_bytes(case):
    """Bytes of a 4-bit page of one head: codes and scales of keys and values."""
    P, D = case["page"], case["head_dim"]
    return P * D + P // min(P, 32) * D + P * (D // 32)


def _seen_in(ctx, n, t, window, sinks):
    """Cached places that a token at depth t behind ctx cached ones sees at most, and new ones of a chain."""
    if not window:
        return ctx, t + 1
    lo = ctx + t - window + 1
    return min(ctx, ctx - max(lo, 0) + min(max(lo, 0), sinks)) if lo < ctx else min(ctx, sinks), min(t + 1, window)


def work(case):
    op = case["op"]
    ctx, new = _spread(case)
    H, D, P = case["kv_heads"], case["head_dim"], case["page"]
    if op in ("pack", "unpack"):
        pages = sum(_whole(case, c) for c in ctx) * H * case["layers"]
        there = pages * (P * D * 4 + _page_bytes(case))
        return {"bytes": there * (2 if op == "pack" else 1), "flops": pages * P * D * 4}
    s, T, B, W, S = 2 if case["dtype"] == "bf16" else 4, case["tokens"], case["batch"], case["window"], case["sinks"]
    each4 = _page_bytes(case) / P if op == "packed" else 0.0
    kv = pairs = 0
    for c, n in zip(ctx, new):
        # every new token sees what the deepest does not, so what is read is what the first one sees
        held = _seen_in(c, n, 0, W, S)[0]
        pk = _whole(case, c) * P if op == "packed" else 0
        near = held if not W else min(c, W - 1)
        in4 = max(0, pk - (c - near)) + (min(S, pk, c - near) if W else 0) if near < c else pk
        kv += H * (in4 * each4 + (max(held - in4, 0) + n) * D * 2 * s)
        if case["tree"]:
            pairs += n * held + n * (n + 1) // 2
        else:
            pairs += sum(sum(_seen_in(c, n, t, W, S)) for t in range(n))
    q = sum(new) * case["q_heads"] * D * s
    out = B * T * case["q_heads"] * (D * s + 4)
    mask = sum(n * n for n in new) if case["tree"] else 0
    return {"bytes": kv + q + out + mask, "flops": 4 * D * case["q_heads"] * pairs}


# ----------------------------------------------------------------------------- the 4-bit format

def _quad(r, i):
    """Row of a block that part i of lane group r holds."""
    return 8 * (r // 2) + r % 2 + 2 * i


def _amount(code):
    """What a scale byte stands for."""
    c = code.to(torch.int32)
    return torch.ldexp(1.0 + (c & 7).float() / 8, (c >> 3) - 19)


def _scale_of(top):
    """The byte of the smallest scale with 7 s >= top (fp32, what 16 bits hold)."""
    m, e = torch.frexp(top.double() / 7)                # m in [1/2, 1)
    eighths = torch.ceil(m * 16).long()                 # 8 .. 16: (1 + k/8) 2^(e - 1)
    code = (e.long() - 1 + 19) * 8 + eighths - 8
    return torch.where(top > 0, code, torch.zeros_like(code)).clamp(0, 255).to(torch.uint8)


def _codes(x, scale):
    """n in -7 .. 7 of x / scale, a half away from 0."""
    y = x.double() / scale.double()
    return (torch.sign(y) * torch.floor(y.abs() + 0.5)).clamp(-7, 7).to(torch.int32)


def _quantised(k, v, N):
    """Codes and scale bytes of pages [..., P, D]: keys by channel over N tokens, values by token over 32 channels."""
    P, D = k.shape[-2:]
    kb, vb = k.unflatten(-2, (P // N, N)), v.unflatten(-1, (D // 32, 32))
    ks, vs = _scale_of(kb.abs().amax(-2)), _scale_of(vb.abs().amax(-1))       # [..., P/N, D], [..., P, D/32]
    kc = _codes(kb, _amount(ks)[..., None, :]).flatten(-3, -2)
    vc = _codes(vb, _amount(vs)[..., None]).flatten(-2, -1)
    return kc, vc, ks, vs


def _words(n):
    """Words of eight codes [..., 8] in the last dimension's place, as int32."""
    c = torch.arange(8, device=n.device)
    u = ((n.long() + 8) << (4 * (c >> 1) + 16 * (c & 1))).sum(-1)
    u = ((u << 3) | (u >> 29)) & 0xFFFFFFFF
    return torch.where(u >= 1 << 31, u - (1 << 32), u).to(torch.int32)


def _order(N, D, device):
    """Rows and columns of a block's words: keys (token, first channel), values (channel, first token)."""
    r = torch.arange(N // 4, device=device)[None, :, None, None]
    x, t = torch.arange(D // 32, device=device)[:, None, None, None], torch.arange(4, device=device)[None, None, :, None]
    i = torch.arange(4, device=device)[None, None, None, :]
    k_row, k_col = _quad(r, i) + 0 * x + 0 * t, 32 * x + 8 * t + 0 * r + 0 * i
    r8, t8 = torch.arange(8, device=device)[None, :, None, None], torch.arange(N // 8, device=device)[None, None, :, None]
    v_row, v_col = 32 * x + _quad(r8, i) + 0 * t8, 8 * t8 + 0 * x + 0 * r8 + 0 * i
    return [y.reshape(-1) for y in (k_row, k_col, v_row, v_col)]


def _pack_pages(k, v):
    """4-bit pages [..., page_bytes] (uint8) of 16-bit ones [..., P, D]."""
    P, D = k.shape[-2:]
    N = min(P, 32)
    kc, vc, ks, vs = _quantised(k, v, N)
    k_row, k_col, v_row, v_col = _order(N, D, k.device)
    c = torch.arange(8, device=k.device)
    kc, vc = kc.unflatten(-2, (P // N, N)), vc.unflatten(-2, (P // N, N))      # [..., P/N, N, D]
    kw = _words(kc[..., k_row[:, None], k_col[:, None] + c])
    vw = _words(vc[..., v_col[:, None] + c, v_row[:, None]])
    vs = vs.unflatten(-2, (P // N, N)).transpose(-1, -2).flatten(-2)
    as_bytes = lambda w: w.contiguous().view(torch.uint8)  # noqa: E731
    return torch.cat([as_bytes(kw), as_bytes(vw), ks, vs], -1).flatten(-2)


def _unpack_pages(data, P, D):
    """Keys and values [..., P, D] (float) that 4-bit pages [..., page_bytes] stand for."""
    N = min(P, 32)
    data = data.unflatten(-1, (P // N, -1))
    half = N * D // 2
    kw, vw = (data[..., a:a + half].contiguous().view(torch.int32).long() & 0xFFFFFFFF for a in (0, half))
    ks = _amount(data[..., 2 * half:2 * half + D])[..., None, :]               # [..., P/N, 1, D]
    vs = _amount(data[..., 2 * half + D:]).unflatten(-1, (D // 32, N))
    vs = vs.transpose(-1, -2).repeat_interleave(32, -1)                        # [..., P/N, N, D]
    k_row, k_col, v_row, v_col = _order(N, D, data.device)
    c = torch.arange(8, device=data.device)
    k = torch.empty(data.shape[:-1] + (N, D), device=data.device)
    v = torch.empty_like(k)

    def numbers(w):
        w = ((w >> 3) | (w << 29)) & 0xFFFFFFFF
        return (((w[..., None] >> (4 * (c >> 1) + 16 * (c & 1))) & 15) - 8).float()

    k[..., k_row[:, None], k_col[:, None] + c] = numbers(kw)
    v[..., v_col[:, None] + c, v_row[:, None]] = numbers(vw)
    return (k * ks).flatten(-3, -2), (v * vs).flatten(-3, -2)


# ----------------------------------------------------------------------------- inputs

class _State:
    pass


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


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


def _table(g, need, slack=3):
    """Pages handed out in random order: the table of `need` pages a request, and the pool's pages."""
    width, total = max(max(need), 1) + slack, sum(need) + slack
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    n = _i32(need).long()
    first, j = torch.cumsum(n, 0) - n, torch.arange(width, device="cuda")[None, :]
    table = torch.where(j < n[:, None], order[(first[:, None] + j).clamp(max=total - 1)], torch.full_like(j, -1, dtype=torch.int32))
    return table.to(torch.int32).contiguous(), total, width, order


def _keys(g, shape, dtype):
    """Normed and rotated keys: some channels an order larger than others, a common direction that heads attend to."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=dtype)
    H, D = shape[-3], shape[-1]
    x += 0.5 * torch.randn((H, 1, D), generator=g, device="cuda", dtype=dtype)
    x *= torch.exp(0.5 * torch.randn((H, 1, D), generator=g, device="cuda")).to(dtype)
    return x


def _in4(g, pages, case):
    """A pool of 4-bit pages [layers, pages, H, page_bytes], made from random keys and values, some layers at a time."""
    made = []
    for _ in range(case.get("layers", 1)):
        shape = (pages, case["kv_heads"], case["page"], case["head_dim"])
        made.append(_pack_pages(_keys(g, shape, torch.bfloat16).float(), torch.randn(shape, generator=g, device="cuda").bfloat16().float()))
    return torch.stack(made)


def prepare(case, seed):
    s, g = _State(), _gen(seed)
    s.case, s.op = dict(case), case["op"]
    ctx, new = _spread(case)
    order = list(range(len(ctx)))
    random.Random(seed).shuffle(order)
    s.ctx, s.new = [ctx[i] for i in order], [new[i] for i in order]
    {"window": _prepare_attend, "packed": _prepare_attend, "pack": _prepare_pack, "unpack": _prepare_unpack}[s.op](s, case, g)
    if own:
        _handles(s, case)
    return s


def _prepare_attend(s, case, g):
    B, T, H, Hq, D, P, dt = (case["batch"], case["tokens"], case["kv_heads"], case["q_heads"], case["head_dim"], case["page"],
                             _dtype(case))
    s.n4 = [_whole(case, c) if s.op == "packed" else 0 for c in s.ctx]
    s.near = [c - n * P for c, n in zip(s.ctx, s.n4)]           # cached tokens in 16 bits
    s.table, s.pages, s.width, _ = _table(g, [-(-(c + n) // P) for c, n in zip(s.near, s.new)])
    s.longest = max(c + n for c, n in zip(s.ctx, s.new))
    shape = (s.pages, H, P, D)
    s.key, s.value = _keys(g, shape, dt), torch.randn(shape, generator=g, device="cuda", dtype=dt)
    if s.op == "packed":
        s.table4, s.pages4, s.width4, _ = _table(g, s.n4)
        s.data = _in4(g, s.pages4, case)
    s.mask = s.depth = None
    if case["tree"]:
        s.mask, s.depth = _trees(g, B, T)
    s.near_t, s.new_t, s.n4_t = _i32(s.near), _i32(s.new) if case["ragged"] else None, _i32(s.n4)
    s.q = torch.randn((B, T, Hq, D), generator=g, device="cuda", dtype=dt)
    s.scale = 1.0 / math.sqrt(D)
    s.out, s.lse = torch.empty_like(s.q), torch.empty((B, T, Hq), dtype=torch.float32, device="cuda")


def _prepare_pack(s, case, g):
    B, P, H, D, layers = case["batch"], case["page"], case["kv_heads"], case["head_dim"], case["layers"]
    need = [-(-c // P) for c in s.ctx]
    s.table, s.pages, s.width, order = _table(g, need)
    shape = (layers, s.pages, H, P, D)
    s.key = _keys(g, shape, torch.bfloat16)
    s.value = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    s.ctx_t, s.n_t = _i32(s.ctx), _i32(need)
    free = [int(p) for p in order[sum(need):].tolist()]
    s.free, s.n_free = _i32(free + [-1] * (s.pages - len(free))), _i32([len(free)])
    # what the requests hold in 4 bits from before, and the stack of the other 4-bit pages
    s.k = [_whole(case, c) for c in s.ctx]
    held = [(3 * b) % 5 for b in range(B)]
    s.pages4, s.width4 = sum(held) + sum(s.k) + 2, max(h + k for h, k in zip(held, s.k)) + 1
    order4, at, rows = torch.randperm(s.pages4, generator=g, device="cuda").tolist(), 0, []
    for h in held:
        rows.append(order4[at:at + h] + [-1] * (s.width4 - h))
        at += h
    s.table4, s.n4_t = _i32(rows), _i32(held)
    s.free4, s.n_free4 = _i32(order4[at:] + [-1] * at), _i32([s.pages4 - at])
    # the places of the pages to come, for reading them back
    s.at_b = torch.tensor([b for b, k in enumerate(s.k) for _ in range(k)], dtype=torch.int64, device="cuda")
    s.at_j = torch.tensor([h + j for h, k in zip(held, s.k) for j in range(k)], dtype=torch.int64, device="cuda")
    s.count = sum(s.k)


def _prepare_unpack(s, case, g):
    n = [_whole(case, c) for c in s.ctx]
    s.count = sum(n)
    s.pages4 = s.count + 3
    s.data = _in4(g, s.pages4, case)
    s.src = torch.randperm(s.pages4, generator=g, device="cuda")[: s.count].to(torch.int32)
    s.pages = s.count
    s.dst = torch.randperm(s.count, generator=g, device="cuda").to(torch.int32)


def _handles(s, case):
    """What a user of the package holds beside the tensors: configurations, workspaces, output buffers."""
    from paper_2609_21827_gb300 import rheo

    s.rheo = rheo
    kw = dict(batch=case["batch"], tokens=case.get("tokens", 1), page_size=case["page"], kv_heads=case["kv_heads"],
              q_heads=case.get("q_heads", case["kv_heads"]), head_dim=case["head_dim"], dtype=case.get("dtype", "bf16"))
    s.cfg = rheo.CacheConfig(pages=s.pages, max_pages=getattr(s, "width", 1), **kw)
    s.ws = rheo.CacheWorkspace(s.cfg)
    if s.op != "window":
        s.cfg4 = rheo.CacheConfig(pages=s.pages4, max_pages=getattr(s, "width4", 1), **kw)
    if s.op in ("window", "packed"):
        s.held = rheo.Pages(s.cfg, block_table=s.table)
        s.held4 = rheo.Pages(s.cfg4, block_table=s.table4, n_pages=s.n4_t) if s.op == "packed" else None
    if s.op == "pack":
        s.held = rheo.Pages(s.cfg, block_table=s.table, n_pages=s.n_t, free_list=s.free, n_free=s.n_free)
        s.held4 = rheo.Pages(s.cfg4, block_table=s.table4, n_pages=s.n4_t, free_list=s.free4, n_free=s.n_free4)
        s.after, s.after4, s.ctx_after = rheo.Pages(s.cfg), rheo.Pages(s.cfg4), torch.empty_like(s.ctx_t)
        s.data = rheo.make_packed(s.cfg4, case["layers"])
        s.dst = torch.arange(s.count, dtype=torch.int32, device="cuda")
    if s.op in ("pack", "unpack"):
        out = rheo.CacheConfig(pages=max(s.count, 1), max_pages=1, **kw)
        s.out_cfg, (s.key_out, s.value_out) = out, rheo.make_cache(out, case["layers"])


# ----------------------------------------------------------------------------- one pass

def run(s):
    return (_RUN_OWN if own else _RUN_PLAIN)[s.op](s)


def _own_window(s):
    c = s.case
    s.rheo.window_attend(s.cfg, s.q, s.key, s.value, s.held, s.near_t, s.out, s.ws, window=c["window"], sinks=c["sinks"],
                         depth=s.depth, new_len=s.new_t, mask=s.mask, lse=s.lse, scale=s.scale)
    return {"out": s.out, "lse": s.lse}


def _own_packed(s):
    c = s.case
    s.rheo.packed_attend(s.cfg, s.cfg4, s.q, s.key, s.value, s.held, s.near_t, s.data[0], s.held4, s.out, s.ws,
                         window=c["window"], sinks=c["sinks"], depth=s.depth, new_len=s.new_t, mask=s.mask, lse=s.lse,
                         scale=s.scale)
    return {"out": s.out, "lse": s.lse}


def _own_pack(s):
    s.rheo.cache_pack(s.cfg, s.cfg4, s.key, s.value, s.data, s.held, s.held4, s.ctx_t, s.ws, keep=s.case["keep"],
                      out=(s.after, s.after4, s.ctx_after))
    src = s.after4.block_table[s.at_b, s.at_j]
    s.rheo.cache_unpack(s.out_cfg, s.cfg4, s.data, s.key_out, s.value_out, src, s.dst, s.ws)
    a, a4 = s.after, s.after4
    return {"key": s.key_out, "value": s.value_out, "ctx": s.ctx_after, "table": a.block_table, "n_pages": a.n_pages,
            "free": a.free_list, "n_free": a.n_free, "table4": a4.block_table, "n_pages4": a4.n_pages, "free4": a4.free_list,
            "n_free4": a4.n_free}


def _own_unpack(s):
    s.rheo.cache_unpack(s.out_cfg, s.cfg4, s.data, s.key_out, s.value_out, s.src, s.dst, s.ws)
    return {"key": s.key_out, "value": s.value_out}


def _plain_attend(s):
    c = s.case
    P, L, H, G, D, B, T = c["page"], s.longest, c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["batch"], \
        c["tokens"]
    at = torch.arange(L, device="cuda")[None, :]
    base = s.n4_t.long()[:, None] * P                              # places before are in 4 bits
    ctx = base + s.near_t.long()[:, None]
    n = torch.full_like(ctx, T) if s.new_t is None else s.new_t.long()[:, None]
    near = (at - base).clamp(min=0)
    held = at < ctx + n
    page = torch.where(held, torch.gather(s.table, 1, (near // P).clamp(max=s.width - 1)).long(), 0)
    here = held[:, None, :, None]
    k = s.key[page, :, near % P].permute(0, 2, 1, 3).float()       # [B, H, L, D]
    v = s.value[page, :, near % P].permute(0, 2, 1, 3).float()
    if s.op == "packed":
        k4, v4 = _unpack_pages(s.data[0], P, D)
        early = at < base
        page4 = torch.where(early, torch.gather(s.table4, 1, (at // P).clamp(max=s.width4 - 1).expand(B, -1)).long(), 0)
        row = (at % P).expand(B, -1)
        early = early[:, None, :, None]
        k = torch.where(early, k4[page4, :, row].permute(0, 2, 1, 3), k)
        v = torch.where(early, v4[page4, :, row].permute(0, 2, 1, 3), v)
    v = torch.where(here, v, 0.0)
    q = s.q.float().reshape(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    x = torch.matmul(q, k.transpose(2, 3)) * s.scale               # [B, H, T*G, L]
    # [B, T, L]: whether new token t sees place l
    t = torch.arange(T, device="cuda")[None, :, None]
    j = at[:, None] - ctx[:, :, None]
    among = j <= t if s.mask is None else torch.gather(s.mask, 2, j.clamp(0, T - 1).expand(-1, T, -1)) != 0
    seen = (j < 0) | (among & (j < n[:, :, None]))
    if c["window"]:
        depth = torch.arange(T, device="cuda")[None, :].expand(B, -1) if s.depth is None else s.depth.long()
        new = torch.gather(depth, 1, j[:, 0].clamp(0, T - 1))
        place = torch.where(j[:, 0] < 0, at, ctx + new)[:, None]   # positions: a drafted token's by its depth
        seen = seen & ((place < c["sinks"]) | ((ctx + depth)[:, :, None] - place < c["window"]))
    seen = seen & (t < n[:, :, None])
    x = torch.where(seen[:, None, :, None, :], x.reshape(B, H, T, G, L), NEG_INF)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == NEG_INF, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, H, T * G, L), v).reshape(B, H, T, G, D)
    o = torch.where(z > 0, o / z, torch.zeros_like(o))
    lse = (m + torch.log(z)).squeeze(-1)
    return {"out": o.permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(s.q.dtype),
            "lse": lse.permute(0, 2, 1, 3).reshape(B, T, H * G)}


def _plain_pack(s):
    c = s.case
    P, D, L = c["page"], c["head_dim"], c["layers"]
    ctx, n, n4 = s.ctx_t.long(), s.n_t.long(), s.n4_t.long()
    k = ((ctx - c["keep"]).clamp(min=0)) // P
    before, total = torch.cumsum(k, 0) - k, s.count
    b, i = s.at_b, torch.arange(total, device="cuda")
    j = i - before[b]
    page, page4 = s.table[b, j].long(), s.free4[s.n_free4.long() - 1 - i]
    data = torch.zeros((L, s.pages4, c["kv_heads"], _page_bytes(c)), dtype=torch.uint8, device="cuda")
    data[:, page4.long()] = _pack_pages(s.key[:, page].float(), s.value[:, page].float())
    # the tables: 4-bit pages come from the top of their stack, 16-bit ones go on theirs, rows move to the front
    table4, free, at = s.table4.clone(), s.free.clone(), torch.arange(s.width, device="cuda")[None, :]
    table4[b, n4[b] + j] = page4
    free[s.n_free.long() + i] = page.to(torch.int32)
    moved = torch.gather(s.table, 1, (at + k[:, None]).clamp(max=s.width - 1))
    table = torch.where(at + k[:, None] < n[:, None], moved, s.table)
    key, value = _unpack_pages(data[:, page4.long()], P, D)
    i32 = torch.int32
    return {"key": key.bfloat16(), "value": value.bfloat16(), "ctx": (ctx - k * P).to(i32), "table": table,
            "n_pages": (n - k).to(i32), "free": free, "n_free": (s.n_free + total).to(i32), "table4": table4,
            "n_pages4": (n4 + k).to(i32), "free4": s.free4, "n_free4": (s.n_free4 - total).to(i32)}


def _plain_unpack(s):
    c = s.case
    k, v = _unpack_pages(s.data[:, s.src.long()], c["page"], c["head_dim"])
    key = torch.empty_like(k, dtype=torch.bfloat16)
    value = torch.empty_like(key)
    key[:, s.dst.long()], value[:, s.dst.long()] = k.bfloat16(), v.bfloat16()
    return {"key": key, "value": value}


_RUN_OWN = {"window": _own_window, "packed": _own_packed, "pack": _own_pack, "unpack": _own_unpack}
_RUN_PLAIN = {"window": _plain_attend, "packed": _plain_attend, "pack": _plain_pack, "unpack": _plain_unpack}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"window": _exact_attend, "packed": _exact_attend, "pack": _exact_pack, "unpack": _exact_unpack}[case["op"]](s, case)


def _exact_values(data, P, D):
    """Keys and values [..., P, D] of 4-bit pages in 64 bits, code by code."""
    lead, N = data.shape[:-1], min(P, 32)
    blocks = data.reshape(-1, P // N, data.shape[-1] // (P // N)).long()
    half, zero = N * D // 2, torch.zeros((), dtype=torch.float64, device=data.device)
    amount = lambda c: (8.0 + c % 8 + zero) * 2.0 ** (c // 8 - 22 + zero)  # noqa: E731
    k = zero.expand(blocks.shape[:2] + (N, D)).clone()
    v = k.clone()
    byte = lambda at: blocks[..., at:at + half].unflatten(-1, (half // 4, 4))  # noqa: E731
    kw, vw = (sum(byte(at)[..., i] * 256 ** i for i in range(4)) for at in (0, half))
    kw, vw = kw.unflatten(-1, (D // 32, N // 4, 4, 4)), vw.unflatten(-1, (D // 32, 8, N // 8, 4))
    for c in range(8):
        bit = (3 + 4 * (c // 2) + 16 * (c % 2)) % 32
        code = lambda w: ((w // 2 ** bit + (w * 2 ** (32 - bit) if bit > 28 else 0)) % 16 - 8).double()  # noqa: E731
        kn, vn = code(kw), code(vw)
        for r in range(8):
            for i in range(4):
                row = 8 * (r // 2) + r % 2 + 2 * i
                for t in range(4):
                    if r < N // 4:
                        k[..., row, 8 * t + c::32] = kn[..., r, t, i]
                    if t < N // 8:
                        v[..., 8 * t + c, row::32] = vn[..., r, t, i]
    k *= amount(blocks[..., 2 * half:2 * half + D])[..., None, :]
    v *= amount(blocks[..., 2 * half + D:].unflatten(-1, (D // 32, N)).transpose(-1, -2)).repeat_interleave(32, -1)
    return k.reshape(*lead, P, D), v.reshape(*lead, P, D)


def _exact_attend(s, c):
    """Request by request: softmax(q k / sqrt(D)) v over the places that a token sees."""
    B, T, H, D, P, W, S = c["batch"], c["tokens"], c["kv_heads"], c["head_dim"], c["page"], c["window"], c["sinks"]
    G = c["q_heads"] // H
    out = torch.zeros((B, T, H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, H * G), NEG_INF, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, near, n4 = s.new[b], s.near[b], s.n4[b]
        ctx, L = s.ctx[b], s.ctx[b] + n
        pages = s.table[b, : -(-(near + n) // P)].long()
        k, v = (x[pages].double().transpose(0, 1).reshape(H, -1, D)[:, : near + n] for x in (s.key, s.value))
        if n4:
            early = [x.transpose(0, 1).reshape(H, -1, D) for x in _exact_values(s.data[0][s.table4[b, :n4].long()], P, D)]
            k, v = torch.cat([early[0], k], 1), torch.cat([early[1], v], 1)
        deep = torch.arange(n, device="cuda") if s.depth is None else s.depth[b, :n].long()
        place = torch.cat([torch.arange(ctx, device="cuda"), ctx + deep])
        seen = torch.ones((n, L), dtype=torch.bool, device="cuda")
        seen[:, ctx:] = torch.ones((n, n), dtype=torch.bool, device="cuda").tril() if s.mask is None else s.mask[b, :n, :n] != 0
        if W:
            seen &= (place < S)[None, :] | (place[None, :] > (ctx + deep)[:, None] - W)
        for h in range(H):
            q = s.q[b, :n, h * G:(h + 1) * G].double()                       # [n, G, D]
            x = (q.reshape(n * G, D) @ k[h].T).reshape(n, G, L) * s.scale
            x.masked_fill_(~seen[:, None, :], NEG_INF)
            w = torch.logsumexp(x, -1, keepdim=True)
            p = torch.exp(x - w).nan_to_num(0.0)
            out[b, :n, h * G:(h + 1) * G] = (p.reshape(n * G, L) @ v[h]).reshape(n, G, D)
            lse[b, :n, h * G:(h + 1) * G] = w[..., 0]
    return {"out": out, "lse": lse}


def _exact_nearest(x, groups):
    """The value of each element after its turn through 4 bits; `groups`: the axis that shares a scale."""
    top = x.abs().amax(groups, keepdim=True)
    steps = torch.tensor([(8 + c % 8) * 2.0 ** (c // 8 - 22) for c in range(256)], dtype=torch.float64, device=x.device)
    s = steps[torch.searchsorted(7 * steps, top.contiguous()).clamp(max=255)]
    low = torch.floor(x.abs() / s)
    n = torch.where(x.abs() - low * s >= (low + 1) * s - x.abs(), low + 1, low).clamp(max=7)
    return torch.copysign(n * s, x)


def _exact_pack(s, c):
    """Request by request: pages off one stack and onto the other, their numbers through 4 bits."""
    P, N = c["page"], min(c["page"], 32)
    table, n, free, top = s.table.tolist(), s.n_t.tolist(), s.free.tolist(), int(s.n_free)
    table4, n4, free4, top4 = s.table4.tolist(), s.n4_t.tolist(), s.free4.tolist(), int(s.n_free4)
    ctx, took = list(s.ctx), []
    for b in range(c["batch"]):
        gone = 0
        while ctx[b] - P >= c["keep"]:
            top4 -= 1
            table4[b][n4[b]] = free4[top4]
            took.append(table[b][gone])
            free[top] = table[b][gone]
            gone, top, n4[b], ctx[b] = gone + 1, top + 1, n4[b] + 1, ctx[b] - P
        n[b] -= gone
        table[b][: n[b]] = table[b][gone: gone + n[b]]
    at = torch.tensor(took, dtype=torch.int64, device="cuda")
    key, value = [], []
    for layer in range(c["layers"]):
        k, v = s.key[layer, at].double(), s.value[layer, at].double()
        key.append(_exact_nearest(k.unflatten(-2, (P // N, N)), -2).flatten(-3, -2).float())
        value.append(_exact_nearest(v.unflatten(-1, (-1, 32)), -1).flatten(-2, -1).float())
    i32 = lambda x: np.array(x, np.int32)  # noqa: E731
    return {"key": torch.stack(key), "value": torch.stack(value), "ctx": i32(ctx), "table": i32(table), "n_pages": i32(n),
            "free": i32(free), "n_free": i32([top]), "table4": i32(table4), "n_pages4": i32(n4), "free4": i32(free4),
            "n_free4": i32([top4])}


def _exact_unpack(s, c):
    """Page by page to its place, a layer at a time."""
    key, value = [], []
    for layer in range(c["layers"]):
        k, v = _exact_values(s.data[layer, s.src.long()], c["page"], c["head_dim"])
        back = torch.argsort(s.dst)
        key.append(k[back].float())
        value.append(v[back].float())
    return {"key": torch.stack(key), "value": torch.stack(value)}
