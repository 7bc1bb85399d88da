"""The operators for long contexts from their definitions in 64 bits, for the tests:
windows, the 4-bit format byte by byte, the tables of cache_pack played through
request by request."""
import functools
import math

import numpy as np
import torch

import cache_reference as ref

MOST = 7 * 1.875 * 2.0 ** 12  # the largest magnitude that 4 bits stand for


# ---- the 4-bit format ---------------------------------------------------------------

def step(code):
    """What a scale byte stands for."""
    code = np.asarray(code, np.int64)
    return (8 + code % 8) * 2.0 ** (code // 8 - 22)


STEPS = step(np.arange(256))


def scale_bytes(top):
    """The smallest scale with 7 s >= top."""
    return np.searchsorted(7 * STEPS, np.minimum(top, MOST)).astype(np.uint8)


def numbers(x, s):
    """The nearest of -7 .. 7 steps, halves away from zero (products of few bits: exact in 64)."""
    n = np.floor(np.abs(x) / s)
    n = np.where(2 * np.abs(x) >= (2 * n + 1) * s, n + 1, n)
    return np.copysign(np.minimum(n, 7), x).astype(np.int64)


def _f(r, i):
    return 8 * (r // 2) + r % 2 + 2 * i


@functools.lru_cache(None)
def word_places(N, D):
    """Rows and columns [words, 8] of a block's words: of the keys (token, channel), of the values (channel, token)."""
    key, value = [], []
    for x in range(D // 32):
        for r in range(N // 4):
            for t in range(4):
                key += [[(_f(r, i), 32 * x + 8 * t + c) for c in range(8)] for i in range(4)]
        for r in range(8):
            for t in range(N // 8):
                value += [[(32 * x + _f(r, i), 8 * t + c) for c in range(8)] for i in range(4)]
    return np.array(key).transpose(2, 0, 1), np.array(value).transpose(2, 0, 1)


BITS = np.array([(3 + 4 * (c // 2) + 16 * (c % 2)) % 32 for c in range(8)], np.uint64)


def _words(codes):
    u = (codes.astype(np.uint64) << BITS).sum(-1)
    return ((u & np.uint64(0xFFFFFFFF)) | (u >> np.uint64(32))).astype(np.uint32)


def _codes(words):
    w = words.astype(np.uint64)
    return (((w | (w << np.uint64(32)))[..., None] >> BITS) & np.uint64(15)).astype(np.int64)


def finite(x):
    """What counts in place of numbers that 4 bits cannot stand for."""
    return np.nan_to_num(np.clip(x, -MOST, MOST), nan=0.0)


def pack_pages(k, v):
    """Bytes [..., page_bytes] of pages [..., P, D] (float64)."""
    P, D = k.shape[-2:]
    N = min(P, 32)
    lead = k.shape[:-2]
    k, v = (finite(x).reshape(-1, P // N, N, D) for x in (k, v))
    ks = scale_bytes(np.abs(k).max(-2))
    vs = scale_bytes(np.abs(v).reshape(*v.shape[:3], D // 32, 32).max(-1)).swapaxes(-1, -2)   # [.., D/32, N]
    kn = numbers(k, step(ks)[..., None, :]) + 8
    vn = numbers(v, np.repeat(step(vs).swapaxes(-1, -2), 32, -1)) + 8
    key, value = word_places(N, D)
    kw, vw = _words(kn[..., key[0], key[1]]), _words(vn[..., value[1], value[0]])
    flat = lambda x: np.ascontiguousarray(x).view(np.uint8).reshape(*x.shape[:2], -1)  # noqa: E731
    return np.concatenate([flat(kw), flat(vw), ks, vs.reshape(*vs.shape[:2], -1)], -1).reshape(*lead, -1)


def unpack_pages(data, P, D):
    """Keys and values [..., P, D] (float64) of bytes [..., page_bytes]."""
    N, lead = min(P, 32), data.shape[:-1]
    x = np.ascontiguousarray(data).reshape(-1, P // N, data.shape[-1] // (P // N))
    half = N * D // 2
    kw, vw = (np.ascontiguousarray(x[..., a:a + half]).view(np.uint32) for a in (0, half))
    ks, vs = x[..., 2 * half:2 * half + D], x[..., 2 * half + D:].reshape(*x.shape[:2], D // 32, N)
    key, value = word_places(N, D)
    k, v = np.zeros(x.shape[:2] + (N, D)), np.zeros(x.shape[:2] + (N, D))
    k[..., key[0], key[1]] = _codes(kw) - 8
    v[..., value[1], value[0]] = _codes(vw) - 8
    k *= step(ks)[..., None, :]
    v *= np.repeat(step(vs).swapaxes(-1, -2), 32, -1)
    return k.reshape(*lead, P, D), v.reshape(*lead, P, D)


# ---- the tables of cache_pack -------------------------------------------------------

def pack_tables(ctx, keep, P, table, n, free, n_free, table4, n4, free4, n_free4, max4):
    """After it: the same, then the pages that moved [(from, to)], whether the stack ran dry, whether a length was bad.
    Plain lists."""
    ctx, n, n4, free = list(ctx), list(n), list(n4), list(free)
    table, table4 = [list(r) for r in table], [list(r) for r in table4]
    moved, dry, short, bad = [], False, False, False
    for b in range(len(ctx)):
        k = max(0, ctx[b] - keep) // P
        if ctx[b] < 0 or n[b] < 0 or n[b] > len(table[b]) or ctx[b] > n[b] * P or n4[b] < 0 or n4[b] + k > max4:
            bad = True
            continue
        dry = dry or k > n_free4 - len(moved)
        if k == 0 or dry:
            short = short or k > 0
            continue
        for j in range(k):
            to = free4[n_free4 - 1 - len(moved)]
            moved.append((table[b][j], to))
            table4[b][n4[b] + j] = to
            free[n_free + len(moved) - 1] = table[b][j]
        table[b][:n[b] - k] = table[b][k:n[b]]
        ctx[b], n[b], n4[b] = ctx[b] - k * P, n[b] - k, n4[b] + k
    return dict(ctx=ctx, table=table, n=n, free=free, n_free=n_free + len(moved), table4=table4, n4=n4, free4=list(free4),
                n_free4=n_free4 - len(moved)), moved, short, bad


# ---- windowed attention -------------------------------------------------------------

def seen(ctx, n, T, mask, depth, window, sinks, device):
    """[n, ctx + n]: what each new token of a request sees."""
    s = torch.ones((n, ctx + n), dtype=torch.bool, device=device)
    s[:, ctx:] = torch.ones((n, n), device=device).tril() > 0 if mask is None else mask[:n, :n] != 0
    if window:
        d = torch.arange(n, device=device) if depth is None else depth[:n].long().clamp(0, T - 1)
        place = torch.cat([torch.arange(ctx, device=device), ctx + d])
        s &= (place < sinks)[None, :] | ((ctx + d)[:, None] - place[None, :] < window)
    return s


def attend(q, lines, ctx, new, mask, depth, window, sinks, scale):
    """out, lse, A and S as cache_reference.attend; lines(b): keys and values [H, ctx + new, D] of request b in 64 bits.
    What a token does not see does not count, whatever it is."""
    B, T, Hq, D = q.shape
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=q.device)
    A, lse = torch.zeros_like(out), torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    S = torch.zeros_like(lse)
    for b in range(B):
        n = int(new[b])
        if n == 0:
            continue
        k, v = lines(b)
        G = Hq // k.shape[0]
        sees = seen(int(ctx[b]), n, T, None if mask is None else mask[b], None if depth is None else depth[b], window, sinks,
                    q.device)
        some = sees.any(1)
        hidden = ~sees.any(0)
        k, v = k.clone(), v.clone()
        k[:, hidden], v[:, hidden] = 0, 0
        for h in range(k.shape[0]):
            qs = q[b, :n, h * G:(h + 1) * G].double()
            x = (qs @ k[h].T * scale).masked_fill(~sees[:, None], -math.inf)
            w = torch.softmax(x, -1)
            w[~some] = 0
            out[b, :n, h * G:(h + 1) * G] = w @ v[h]
            A[b, :n, h * G:(h + 1) * G] = w @ v[h].abs()
            lse[b, :n, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            S[b, :n, h * G:(h + 1) * G] = (qs.abs() @ k[h].abs().T).amax(-1) * abs(scale)
    return out, lse, A, S


def tree_masks(B, T, g):
    """Ancestor masks of random trees and the nodes' depths."""
    m = torch.zeros((B, T, T), dtype=torch.uint8)
    for b in range(B):
        for i in range(T):
            if i:
                m[b, i] = m[b, int(torch.randint(max(0, i - 7), i, (1,), generator=g))]
            m[b, i, i] = 1
    return m.cuda(), (m.sum(2) - 1).to(torch.int32).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Problem:
    """Requests with n4 packed pages and `near` tokens in 16 bits behind them (n4 None: no packed part), and one call of
    window_attend or packed_attend.  What no request holds is not a number; so is what lies outside every window."""

    def __init__(self, rheo, near, new, T, Hq, H, D, P, dtype="bf16", n4=None, tree=False, window=0, sinks=0, layout="heads",
                 seed=0, spread=1.0, with_depth=True):
        g, gd = torch.Generator().manual_seed(2000 + seed), torch.Generator(device="cuda").manual_seed(seed)
        self.rheo = rheo
        B = len(near)
        self.near, self.new, self.n4 = list(near), [T] * B if new is None else list(new), n4
        self.given_new, self.T, self.window, self.sinks = new is not None, T, window, sinks
        self.ctx = [c + (0 if n4 is None else n4[b] * P) for b, c in enumerate(near)]
        self.mask, depth = tree_masks(B, T, g) if tree else (None, None)
        self.depth = depth if with_depth else None
        lens = [c + n for c, n in zip(self.near, self.new)]
        kw = dict(batch=B, tokens=T, page_size=P, q_heads=Hq, kv_heads=H, head_dim=D, dtype=dtype)

        def handed_out(need):
            pages, width = sum(need) + 3, max(max(need), 1) + 2
            order = torch.randperm(pages, generator=g).tolist()
            table, at = torch.full((B, width), -2 ** 30, dtype=torch.int32), 0
            for b, n in enumerate(need):
                table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
                at += n
            return table, pages, width

        table, pages, width = handed_out([-(-n // P) for n in lens])
        self.cfg = rheo.CacheConfig(pages=pages, max_pages=width, **kw)
        self.table = table.cuda()
        dt = self.cfg.torch_dtype
        rnd = lambda *s: torch.randn(s, generator=gd, device="cuda").to(dt)  # noqa: E731
        if layout == "heads":
            self.key, self.value = rnd(pages, H, P, D), rnd(pages, H, P, D)
            self.q, self.out = (spread * rnd(B, T, Hq, D)).to(dt), torch.full((B, T, Hq, D), 3.0, dtype=dt, device="cuda")
        else:
            pool = rnd(pages, P, H, 2, D + 8 * (4 // dt.itemsize))
            self.key, self.value = (pool[:, :, :, i, :D].transpose(1, 2) for i in (0, 1))
            self.q = (spread * rnd(B, T, Hq + 2 * H, D)).to(dt)[:, :, :Hq]
            self.out = torch.full((B, Hq, T, D), 3.0, dtype=dt, device="cuda").transpose(1, 2)
        held = torch.zeros((pages, P), dtype=torch.bool)
        for b, n in enumerate(lens):
            for x in range(n):
                held[int(table[b, x // P]), x % P] = True
        hole = ~held.cuda()
        for c in (self.key, self.value):
            c.transpose(1, 2)[hole] = math.nan
        self.held = rheo.Pages(self.cfg, block_table=self.table)
        self.scale = D ** -0.5
        self.lse = torch.full((B, T, Hq), 3.0, device="cuda")
        self.ws = rheo.CacheWorkspace(self.cfg)
        if n4 is not None:
            table4, pages4, width4 = handed_out(n4)
            self.cfg4 = rheo.CacheConfig(pages=pages4, max_pages=width4, **kw)
            x = [torch.randn((pages4, H, P, D), generator=gd, device="cuda").bfloat16().double().cpu().numpy() for _ in range(2)]
            x[0] *= np.exp(np.random.RandomState(seed).randn(1, H, 1, D))
            data = pack_pages(*x)
            if layout == "heads":
                self.data = torch.from_numpy(data).cuda()
            else:  # heads before pages, padded
                wide = torch.full((H, pages4, data.shape[-1] + 48), 0xFF, dtype=torch.uint8, device="cuda")
                self.data = wide[:, :, :data.shape[-1]].transpose(0, 1)
                self.data.copy_(torch.from_numpy(data))
            self.table4 = table4.cuda()
            self.held4 = rheo.Pages(self.cfg4, block_table=self.table4, n_pages=i32(n4))

    def lines(self, b):
        P = self.cfg.page_size
        n = self.near[b] + self.new[b]
        k, v = (ref.lines(c, self.table[b], n, P) for c in (self.key, self.value))
        if self.n4 is not None and self.n4[b]:
            data = self.data[self.table4[b, :self.n4[b]].long()].cpu().numpy()
            early = [torch.from_numpy(x).cuda().transpose(0, 1).reshape(k.shape[0], -1, k.shape[2])
                     for x in unpack_pages(data, P, k.shape[2])]
            k, v = torch.cat([early[0], k], 1), torch.cat([early[1], v], 1)
        return k, v

    def run(self, stream=None):
        kw = dict(window=self.window, sinks=self.sinks, depth=self.depth, new_len=i32(self.new) if self.given_new else None,
                  mask=self.mask, lse=self.lse, scale=self.scale, stream=stream)
        a = (self.q, self.key, self.value, self.held, i32(self.near))
        if self.n4 is None:
            self.rheo.window_attend(self.cfg, *a, self.out, self.ws, **kw)
        else:
            self.rheo.packed_attend(self.cfg, self.cfg4, *a, self.data, self.held4, self.out, self.ws, **kw)
        return self.out, self.lse

    def check(self, stream=None):
        out, lse = self.run(stream)
        assert self.rheo.scratch_status(self.ws) == 0
        o, w, A, S = attend(self.q, self.lines, self.ctx, self.new, self.mask, self.depth, self.window, self.sinks, self.scale)
        L = max(c + n for c, n in zip(self.ctx, self.new))
        e, el = ref.attend_bounds(o, w, A, S, self.cfg.head_dim, L, self.cfg.dtype == "bf16")
        none = w == -math.inf
        assert torch.equal(lse == -math.inf, none) and not out[none].any()
        assert not torch.isnan(out).any()
        err = (out.double() - o).abs()
        assert (err <= e).all(), f"out: {float((err / e).max()):.3g} of the bound"
        err = (lse.double() - w).abs()[~none]
        assert (err <= el[~none]).all(), f"lse: {float((err / el[~none]).max()):.3g} of the bound"
        return out, lse
