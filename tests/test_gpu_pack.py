"""Pages into 4 bits and back: every byte and every table entry against the
definitions (long_reference.py)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import long_reference as lr

pytestmark = pytest.mark.gpu
i32 = lr.i32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


class Caches:
    """Requests with ctx tokens in 16 bits and n4 packed pages, random pages, and what is free of both pools."""

    def __init__(self, ctx, n4, P, H=2, D=64, layers=1, free4=None, layout="heads", seed=0, spare=5):
        g, gd = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
        B, n = len(ctx), [-(-c // P) for c in ctx]
        want4 = sum(n) + spare if free4 is None else free4
        kw = dict(batch=B, tokens=3, page_size=P, q_heads=H, kv_heads=H, head_dim=D)
        self.cfg = rheo.CacheConfig(pages=sum(n) + spare, max_pages=max(n) + 2, **kw)
        self.cfg4 = rheo.CacheConfig(pages=sum(n4) + want4, max_pages=max(a + b for a, b in zip(n, n4)) + 1, **kw)
        self.P, self.layers = P, layers

        def tables(cfg, held):
            order = torch.randperm(cfg.pages, generator=g).tolist()
            rows, at = [], 0
            for h in held:
                rows.append(order[at:at + h] + [-7] * (cfg.max_pages - h))
                at += h
            return rows, order[at:] + [-9] * at, cfg.pages - at

        self.table, self.free, self.n_free = tables(self.cfg, n)
        self.table4, self.free4, self.n_free4 = tables(self.cfg4, n4)
        self.ctx, self.n, self.n4 = list(ctx), n, list(n4)
        shape = (layers, self.cfg.pages, H, P, D)
        rnd = lambda *s: torch.randn(s, generator=gd, device="cuda")  # noqa: E731
        k, v = rnd(*shape) * torch.exp(2 * rnd(H, 1, D)), rnd(*shape) * torch.exp(2 * rnd(layers, self.cfg.pages, H, P, 1))
        if layout == "heads":
            self.key, self.value = k.bfloat16(), v.bfloat16()
            self.data = rheo.make_packed(self.cfg4, layers)
        else:  # layers innermost of the pages, tokens before heads, keys and values side by side; packed heads first
            pool = torch.zeros((self.cfg.pages, layers, P, H, 2, D), dtype=torch.bfloat16, device="cuda")
            self.key, self.value = (pool[:, :, :, :, i].permute(1, 0, 3, 2, 4) for i in (0, 1))
            self.key.copy_(k)
            self.value.copy_(v)
            nbytes = rheo.packed_page_bytes(self.cfg4)
            self.data = torch.zeros((H, layers, self.cfg4.pages, nbytes + 16), dtype=torch.uint8,
                                    device="cuda")[..., :nbytes].permute(1, 2, 0, 3)
        self.data.fill_(0x5A)
        self.ws = rheo.CacheWorkspace(self.cfg)

    def state(self):
        pages = rheo.Pages(self.cfg, block_table=i32(self.table), n_pages=i32(self.n), free_list=i32(self.free),
                           n_free=i32([self.n_free]))
        pages4 = rheo.Pages(self.cfg4, block_table=i32(self.table4), n_pages=i32(self.n4), free_list=i32(self.free4),
                            n_free=i32([self.n_free4]))
        return pages, pages4, i32(self.ctx)

    def pack(self, keep=0, in_place=True, stream=None):
        """The call, its state after it as lists, and the packed bytes."""
        pages, pages4, ctx = self.state()
        out = None if in_place else (rheo.Pages(self.cfg), rheo.Pages(self.cfg4), torch.zeros_like(ctx))
        rheo.cache_pack(self.cfg, self.cfg4, self.key, self.value, self.data, pages, pages4, ctx, self.ws, keep=keep, out=out,
                        stream=stream)
        torch.cuda.synchronize()
        if not in_place:
            before = self.state()
            for a, b in ((pages, before[0]), (pages4, before[1])):
                assert all(torch.equal(getattr(a, f), getattr(b, f)) for f in ("block_table", "n_pages", "free_list", "n_free"))
            assert torch.equal(ctx, before[2])
            pages, pages4, ctx = out
        return self.lists(pages, pages4, ctx)

    @staticmethod
    def lists(pages, pages4, ctx):
        return dict(ctx=ctx.tolist(), table=pages.block_table.tolist(), n=pages.n_pages.tolist(), free=pages.free_list.tolist(),
                    n_free=int(pages.n_free), table4=pages4.block_table.tolist(), n4=pages4.n_pages.tolist(),
                    free4=pages4.free_list.tolist(), n_free4=int(pages4.n_free))

    def check(self, keep=0, in_place=True, status=0):
        before = self.data.cpu().numpy().copy()
        got = self.pack(keep, in_place)
        want, moved, short, bad = lr.pack_tables(self.ctx, keep, self.P, self.table, self.n, self.free, self.n_free, self.table4,
                                                 self.n4, self.free4, self.n_free4, self.cfg4.max_pages)
        st = (rheo.STATUS_NO_PAGES if short else 0) | (rheo.STATUS_BAD_LENGTH if bad else 0) | status
        assert rheo.scratch_status(self.ws) == st
        assert got == want
        if moved:
            src, dst = (list(x) for x in zip(*moved))
            k, v = (c[:, src].double().cpu().numpy() for c in (self.key, self.value))
            before[:, dst] = lr.pack_pages(k, v)
        assert (self.data.cpu().numpy() == before).all()
        return want, moved


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("H,D,layers", [(1, 64, 1), (2, 128, 3), (5, 64, 2)])
@pytest.mark.parametrize("layout", ["heads", "mixed"])
def test_every_byte_and_table(P, H, D, layers, layout):
    ctx = [0, 1, P - 1, P, P + 1, 5 * P, 3 * P + 7, 2 * P]
    for in_place in (True, False):
        Caches(ctx, [0, 3, 1, 0, 2, 1, 0, 4], P, H, D, layers, layout=layout, seed=P + D).check(in_place=in_place)


@pytest.mark.parametrize("keep", [0, 1, 15, 16, 17, 40, 10 ** 9, 2 ** 31 - 1])
def test_tokens_that_stay(keep):
    Caches([0, 16, 17, 31, 33, 80, 200], [0] * 7, 16, seed=keep % 91).check(keep, in_place=keep % 2 == 0)


@pytest.mark.parametrize("B", [1, 2, 255, 256, 257, 700, 4096])
def test_many_requests(B):
    """More than a CTA's threads; every fifth packs nothing."""
    Caches([(7 * b) % 50 if b % 5 else 3 for b in range(B)], [b % 3 for b in range(B)], 16, 1, 64, seed=B).check(5, B % 2 == 0)


def test_rows_of_tables_longer_than_a_cta():
    """Hundreds of pages move to the front of a row, in place, by fewer and by more places than a CTA has threads."""
    P = 16
    c = Caches([P * 900 + 5, P * 700], [0, 2], P, 1, 64, seed=3)
    for keep in (P * 890, P * 600, P * 300, 0):
        for in_place in (True, False):
            c.check(keep, in_place)


@pytest.mark.parametrize("free4", [0, 1, 4, 5, 9, 10, 11])
def test_a_stack_that_runs_dry(free4):
    """Requests of 4, 0, 1, 5, 0 and 2 pages."""
    for in_place in (True, False):
        Caches([64, 3, 17, 80, 0, 33], [1, 0, 0, 2, 0, 0], 16, free4=free4, seed=free4).check(in_place=in_place)


def test_bad_lengths_leave_requests_as_they_are():
    c = Caches([64, 64, 64, 64, 64, 64], [0] * 6, 16, seed=1)
    c.ctx = [64, -1, 65, 64, 40, 2 ** 31 - 1]
    c.n4 = [0, 0, 0, c.cfg4.max_pages - 3, 0, 0]    # the fourth's table has room for three of its four pages
    c.check()
    c = Caches([64, 64, 64, 64], [0] * 4, 16, seed=1)
    c.n, c.n4 = [4, -1, 2 ** 31 - 1, 4], [0, 0, 0, -5]
    c.check()


def test_bad_pages_are_left_out():
    for where, wrong in (("table", -1), ("table", 10 ** 6), ("free4", -1), ("free4", 2 ** 31 - 1)):
        c = Caches([64, 48], [0, 0], 16, seed=2)
        before = c.data.cpu().numpy().copy()
        if where == "table":
            c.table[0][1] = wrong
        else:
            c.free4[c.n_free4 - 2] = wrong
        got = c.pack()
        assert rheo.scratch_status(c.ws) == rheo.STATUS_BAD_INDEX
        want, moved, _, _ = lr.pack_tables(c.ctx, 0, 16, c.table, c.n, c.free, c.n_free, c.table4, c.n4, c.free4, c.n_free4,
                                           c.cfg4.max_pages)
        assert got == want
        fine = [m for m in moved if wrong not in m]
        assert len(fine) == len(moved) - 1
        src, dst = (list(x) for x in zip(*fine))
        before[:, dst] = lr.pack_pages(*(x[:, src].double().cpu().numpy() for x in (c.key, c.value)))
        assert (c.data.cpu().numpy() == before).all()


def test_stacks_of_wrong_height_set_a_bit():
    c = Caches([64, 48], [0, 0], 16, seed=2)
    good = c.n_free4
    c.n_free4 = -3
    assert c.pack()["n4"] == [0, 0]
    assert rheo.scratch_status(c.ws) == rheo.STATUS_INTERNAL | rheo.STATUS_NO_PAGES
    c.n_free4, c.n_free = good, c.cfg.pages + 4
    c.pack()
    assert rheo.scratch_status(c.ws) == rheo.STATUS_INTERNAL


@pytest.mark.parametrize("P", [16, 64])
def test_ends_and_halves(P):
    """Magnitudes of exactly seven steps, numbers exactly between two codes, zeros, the smallest and the largest scales,
    and every one of the 16-bit numbers that are finite and in range."""
    D, pages = 64, 80
    c = Caches([P * pages], [0], P, 1, D, seed=4)
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).float()
    every = every[torch.isfinite(every) & (every.abs() <= lr.MOST)]
    g = torch.Generator().manual_seed(1)
    x = every[torch.randint(0, len(every), (c.cfg.pages, 1, P, D), generator=g)]
    s = torch.tensor(lr.STEPS)[torch.randint(8, 256, (c.cfg.pages, 1, P, D), generator=g)].float()
    ties = (torch.randint(-7, 7, s.shape, generator=g) + 0.5) * s[:, :, :1, :1]
    which = torch.randint(0, 4, (c.cfg.pages, 1, 1, 1), generator=g)
    k = torch.where(which == 0, x, torch.where(which == 1, ties, torch.where(which == 2, 7 * s[:, :, :1], 0.0 * x)))
    k[which.expand_as(k)[:, :, :, :] == 1] = ties[which.expand_as(k) == 1]
    k[:, :, 0][which[:, :, 0].expand_as(k[:, :, 0]) == 1] = (7 * s[:, :, :1, :1]).expand_as(k)[:, :, 0][
        which[:, :, 0].expand_as(k[:, :, 0]) == 1]
    k = k.clamp(-lr.MOST, lr.MOST)
    c.key.copy_(k[None])
    c.value.copy_(k.transpose(2, 3).reshape(k.shape)[None])
    assert (c.key.float().cpu()[0] == k).all()      # all of it is held exactly
    c.check()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 54016.0, -3e38])
@pytest.mark.parametrize("P,at", [(16, (0, 0)), (32, (31, 63)), (64, (40, 17))])
def test_numbers_that_no_code_stands_for(bad, P, at):
    for which in (0, 1):
        c = Caches([P, P, 3 * P], [0, 1, 0], P, 2, 64, 2, seed=5)
        (c.key, c.value)[which][1, c.table[2][1], 1, at[0], at[1]] = bad
        c.check(status=rheo.STATUS_BAD_VALUE)


def test_a_page_of_nothing_but_bad_numbers():
    c = Caches([32, 32], [0, 0], 32, 1, 64, seed=5)
    c.key[:], c.value[:] = math.nan, -math.inf
    c.check(status=rheo.STATUS_BAD_VALUE)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("layout", ["heads", "mixed"])
@pytest.mark.parametrize("D", [64, 128])
def test_unpack(P, layout, D):
    """Any bytes; pages in any order, some left out."""
    H, layers, n = 3, 2, 7
    c = Caches([P * 9], [0], P, H, D, layers, layout=layout, seed=6)
    g = torch.Generator().manual_seed(P)
    nbytes = c.data.shape[-1]
    c.data.copy_(torch.randint(0, 256, (layers, c.cfg4.pages, H, nbytes), generator=g).to(torch.uint8))
    src = torch.randperm(c.cfg4.pages, generator=g)[:n].tolist()
    dst = torch.randperm(c.cfg.pages, generator=g)[:n].tolist()
    k, v = lr.unpack_pages(c.data.cpu().numpy(), P, D)
    want = [x.double().cpu() for x in (c.key, c.value)]
    src[2], dst[4] = -1, -1
    for a, b in zip(src, dst):
        if a >= 0 and b >= 0:
            want[0][:, b], want[1][:, b] = torch.from_numpy(k[:, a]), torch.from_numpy(v[:, a])
    rheo.cache_unpack(c.cfg, c.cfg4, c.data, c.key, c.value, i32(src), i32(dst), c.ws)
    assert rheo.scratch_status(c.ws) == 0
    assert torch.equal(c.key.double().cpu(), want[0]) and torch.equal(c.value.double().cpu(), want[1])
    for wrong in (-2, c.cfg4.pages, 2 ** 31 - 1):
        rheo.cache_unpack(c.cfg, c.cfg4, c.data, c.key, c.value, i32([wrong, src[0]]), i32([dst[0], dst[0]]), c.ws)
        assert rheo.scratch_status(c.ws) == rheo.STATUS_BAD_INDEX
        rheo.cache_unpack(c.cfg, c.cfg4, c.data, c.key, c.value, i32([src[0]]), i32([wrong if wrong < 0 else c.cfg.pages]), c.ws)
        assert rheo.scratch_status(c.ws) == rheo.STATUS_BAD_INDEX
    rheo.cache_unpack(c.cfg, c.cfg4, c.data, c.key, c.value, i32([]), i32([]), c.ws)
    assert torch.equal(c.key.double().cpu(), want[0]) and torch.equal(c.value.double().cpu(), want[1])


def test_one_packed_page_into_many():
    """The same page may be unpacked twice in a call, to different places."""
    c = Caches([32 * 4], [0], 32, 2, 64, seed=7)
    _, moved = c.check()
    src = [moved[1][1]] * 3
    rheo.cache_unpack(c.cfg, c.cfg4, c.data, c.key, c.value, i32(src), i32([0, 2, 3]), c.ws)
    k, _ = lr.unpack_pages(c.data[:, src[0]].cpu().numpy(), 32, 64)
    assert all(torch.equal(c.key[:, p].double().cpu(), torch.from_numpy(k)) for p in (0, 2, 3))


def test_cycle_by_cycle_in_a_graph_and_on_a_stream():
    """A captured call that packs in place, replayed as lengths grow; then a request ends and gives its packed pages back."""
    P, B = 16, 3
    c = Caches([70, 5, 33], [0, 0, 0], P, 2, 64, seed=8, spare=40)
    pages, pages4, ctx = c.state()
    call = lambda s=None: rheo.cache_pack(c.cfg, c.cfg4, c.key, c.value, c.data, pages, pages4, ctx, c.ws, keep=20,  # noqa: E731
                                          stream=s)
    state = c.lists(pages, pages4, ctx)
    play = lambda s: lr.pack_tables(s["ctx"], 20, P, s["table"], s["n"], s["free"], s["n_free"], s["table4"], s["n4"],  # noqa: E731
                                    s["free4"], s["n_free4"], c.cfg4.max_pages)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.synchronize()
    want, _, _, _ = play(state)
    assert c.lists(pages, pages4, ctx) == want
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    assert c.lists(pages, pages4, ctx) == want
    plan, ws = rheo.CachePlan(c.cfg), rheo.CacheWorkspace(c.cfg)
    for grow in ([3, 3, 0], [3, 3, 2], [1, 0, 3], [3, 3, 3], [3, 3, 3], [3, 3, 3], [3, 3, 3]):
        rheo.cache_reserve(c.cfg, ctx, pages, plan, ws, new_len=i32(grow))
        assert rheo.scratch_status(ws) == 0
        ctx += i32(grow)
        state = c.lists(pages, pages4, ctx)
        graph.replay()
        torch.cuda.synchronize()
        want, _, _, _ = play(state)
        assert c.lists(pages, pages4, ctx) == want
        assert rheo.scratch_status(c.ws) == 0
    held = pages4.n_pages.clone()
    assert int(held[0]) > 0 and int(held[2]) > 0
    left = held * P
    left[0] = 0
    rheo.cache_reserve(c.cfg4, left, pages4, rheo.CachePlan(c.cfg4), ws, new_len=i32([0] * B))
    assert rheo.scratch_status(ws) == 0
    assert pages4.n_pages.tolist() == [0, int(held[1]), int(held[2])]
    assert int(pages4.n_free) == want["n_free4"] + int(held[0])


def test_caches_past_32_bits():
    """Pages whose numbers lie more than 2^32 bytes from the first."""
    P, H, D = 128, 8, 128
    far = 2 ** 32 // (P * H * D * 2) + 3
    kw = dict(batch=1, tokens=1, page_size=P, q_heads=H, kv_heads=H, head_dim=D)
    cfg, cfg4 = rheo.CacheConfig(pages=far + 2, max_pages=4, **kw), rheo.CacheConfig(pages=4 * far + 3, max_pages=4, **kw)
    key, value = rheo.make_cache(cfg)
    data = rheo.make_packed(cfg4)
    ws = rheo.CacheWorkspace(cfg)
    for p in (far, far + 1):
        key[0, p], value[0, p] = torch.randn((H, P, D), device="cuda"), torch.randn((H, P, D), device="cuda")
    pages = rheo.Pages(cfg, block_table=i32([[far + 1, far, -1, -1]]), n_pages=i32([2]), n_free=i32([far]))
    free4 = i32([0] * (4 * far + 1) + [4 * far, 4 * far + 2])
    pages4 = rheo.Pages(cfg4, free_list=free4)
    want = lr.pack_pages(*(x[0, [far + 1, far]].double().cpu().numpy() for x in (key, value)))
    ctx = i32([2 * P])
    rheo.cache_pack(cfg, cfg4, key, value, data, pages, pages4, ctx, ws)
    assert (data[0, [4 * far + 2, 4 * far]].cpu().numpy() == want).all()
    rheo.cache_unpack(cfg, cfg4, data, key, value, i32([4 * far]), i32([far + 1]), ws)
    assert rheo.scratch_status(ws) == 0
    assert torch.equal(key[0, far + 1].double().cpu(), torch.from_numpy(lr.unpack_pages(want[1], P, D)[0]))
