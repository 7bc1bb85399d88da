"""The paged cache on the GPU: block tables and slots from lengths, query/key
norms with rotation and the store, and the commit of the accepted path, each
against its definition in 64 bits (tests/cache_reference.py)."""
import pytest
import torch

from paper_2609_21827_gb300 import build, rheo
import cache_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    build.build()


def _cfg(**kw):
    base = dict(batch=2, tokens=5, pages=64, page_size=16, max_pages=16, q_heads=4, kv_heads=2, head_dim=64, dtype="f32")
    base.update(kw)
    return rheo.CacheConfig(**base)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(cfg, lens, g):
    """Random distinct pages for `lens` tokens a request; the entries behind them point far out of the pool."""
    order = torch.randperm(cfg.pages, generator=g).tolist()
    table, at = torch.full((cfg.batch, cfg.max_pages), 2 ** 30, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        need = -(-n // cfg.page_size)
        table[b, :need] = torch.tensor(order[at:at + need], dtype=torch.int32)
        at += need
    assert at <= cfg.pages
    return table.cuda()


# ---------------------------------------------------------------- reserve

RESERVE = [
    # ctx, new, pages, owned by each request beforehand
    dict(ctx=[0], new=[1], pages=1, owned=[0]),
    dict(ctx=[15, 16, 17, 0], new=[1, 1, 16, 0], pages=12, owned=[1, 1, 2, 3]),
    dict(ctx=[100, 0, 31, 64, 5], new=[9, 0, 1, 0, 9], pages=40, owned=[3, 7, 2, 6, 0]),
    # the pool runs dry at the third request; the fourth lacks nothing and is served
    dict(ctx=[40, 40, 200, 10, 40], new=[9, 9, 9, 6, 9], pages=10, owned=[0, 0, 0, 1, 0]),
    # pages that are given back serve the others in the same call
    dict(ctx=[0, 120, 0, 60], new=[0, 8, 0, 4], pages=12, owned=[6, 0, 6, 0]),
    # lengths past the table, negative, and more new tokens than the call has
    dict(ctx=[250, -1, 3, 30], new=[9, 3, 10, 4], pages=20, owned=[1, 1, 1, 1]),
    dict(ctx=[7 * b % 200 for b in range(600)], new=[b % 10 for b in range(600)], pages=9000,
         owned=[(5 * b) % 12 for b in range(600)]),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("with_depth", [False, True])
@pytest.mark.parametrize("case", range(len(RESERVE)))
def test_reserve_matches_the_stack(case, with_depth, in_place):
    c = RESERVE[case]
    B, T, P, W = len(c["ctx"]), 9, 16, 16
    cfg = _cfg(batch=B, tokens=T, pages=c["pages"], page_size=P, max_pages=W)
    g = torch.Generator().manual_seed(case)
    order = torch.randperm(c["pages"], generator=g).tolist()
    table, at = [], 0
    for n in c["owned"]:
        table.append(order[at:at + n] + [-7] * (W - n))
        at += n
    free = order[at:]
    n_free = len(free)
    free = free + [-9] * (c["pages"] - n_free)
    depth = torch.randint(0, 6, (B, T), generator=g).tolist() if with_depth else None
    want = ref.reserve(c["ctx"], c["new"], depth, table, c["owned"], free, n_free, P, T, W)

    before = rheo.Pages(cfg, block_table=_i32(table), n_pages=_i32(c["owned"]), free_list=_i32(free), n_free=_i32([n_free]))
    keep = [x.clone() for x in (before.block_table, before.n_pages, before.free_list, before.n_free)]
    after = before if in_place else rheo.Pages(cfg)
    plan, ws = rheo.CachePlan(cfg), rheo.CacheWorkspace(cfg)
    for again in range(2):  # out of place the call can be repeated: its tickets are clean
        if again and in_place:
            break
        rheo.cache_reserve(cfg, _i32(c["ctx"]), before, plan, ws, new_len=_i32(c["new"]),
                           depth=_i32(depth) if with_depth else None, out=None if in_place else after)
        status = rheo.scratch_status(ws)
        assert status == (rheo.STATUS_NO_PAGES if want[6] else 0) | (rheo.STATUS_BAD_LENGTH if want[7] else 0)
        assert after.block_table.tolist() == want[0]
        assert after.n_pages.tolist() == want[1]
        assert after.free_list.tolist() == want[2]
        assert after.n_free.tolist() == [want[3]]
        assert plan.slot.tolist() == want[4]
        assert plan.position.tolist() == want[5]
    if not in_place:
        for x, y in zip(keep, (before.block_table, before.n_pages, before.free_list, before.n_free)):
            assert torch.equal(x, y)


def test_reserve_from_an_empty_pool_cycle_by_cycle():
    """Requests that grow by what they accept, end, and start anew never share a page."""
    cfg = _cfg(batch=3, tokens=7, pages=30, max_pages=8, page_size=16)
    pages, plan, ws = rheo.Pages(cfg), rheo.CachePlan(cfg), rheo.CacheWorkspace(cfg)
    ctx = [0, 0, 0]
    for cycle in range(40):
        new = [7, 7, 7]
        if cycle % 9 == 8:
            ctx[cycle % 3], new[cycle % 3] = 0, 0
        rheo.cache_reserve(cfg, _i32(ctx), pages, plan, ws, new_len=_i32(new))
        assert rheo.scratch_status(ws) == 0
        held = [pages.block_table[b, :n].tolist() for b, n in enumerate(pages.n_pages.tolist())]
        flat = sum(held, []) + pages.free_list[: int(pages.n_free)].tolist()
        assert sorted(flat) == list(range(30))
        for b in range(3):
            for t in range(new[b]):
                page, row = ref.place(held[b], ctx[b] + t, 16)
                assert int(plan.slot[b, t]) == page * 16 + row
        ctx = [min(c + (1 + (cycle + b) % 4 if new[b] else 0), 120) for b, c in enumerate(ctx)]


def test_tables_that_have_moved_are_found_again():
    """Storage exchanged under a tensor that an earlier call has seen."""
    cfg = _cfg(batch=1, tokens=4, pages=8, max_pages=4)
    pages, plan, ws = rheo.Pages(cfg), rheo.CachePlan(cfg), rheo.CacheWorkspace(cfg)
    rheo.cache_reserve(cfg, _i32([0]), pages, plan, ws)
    old, other = pages.block_table.clone(), torch.full((1, 4), 5, dtype=torch.int32, device="cuda")
    kept = pages.block_table.untyped_storage()  # not freed, so that the new one lies elsewhere
    pages.block_table.data = other
    plan.slot.data = torch.zeros_like(plan.slot)
    rheo.cache_reserve(cfg, _i32([4]), pages, plan, ws)
    assert plan.slot.tolist() == [[5 * 16 + 4 + t for t in range(4)]] and old.tolist() != other.tolist()
    pages.block_table.data = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    with pytest.raises(rheo.RheoError):
        rheo.cache_reserve(cfg, _i32([4]), pages, plan, ws)
    assert kept.nbytes() and rheo.scratch_status(ws) == 0


# ---------------------------------------------------------------- qk_norm_rope

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot,Hq,H", [(64, 64, 4, 2), (128, 128, 32, 8), (128, 24, 5, 5), (64, 32, 3, 1), (128, 0, 2, 1),
                                        (64, 8, 20, 4)])
@pytest.mark.parametrize("interleaved,norm,layout", [(False, "both", "packed"), (True, "q", "heads"),
                                                     (False, "none", "in place"), (True, "both", "pairs")])
def test_norm_rope_and_store(dtype, D, rot, Hq, H, interleaved, norm, layout):
    B, T, P = 3, 4, 16
    cfg = _cfg(batch=B, tokens=T, pages=20, page_size=P, max_pages=6, q_heads=Hq, kv_heads=H, head_dim=D, dtype=dtype)
    dt, g = cfg.torch_dtype, torch.Generator(device="cuda").manual_seed(D + rot + Hq)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    qkv = (3 * rnd(B, T, Hq + 2 * H, D)).to(dt)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    if layout == "heads":  # [B, heads, T, D] products
        q, k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v))
    qw = (1 + 0.3 * rnd(D)).to(dt) if norm in ("both", "q") else None
    kw = (1 + 0.3 * rnd(D)).to(dt) if norm == "both" else None
    positions = 700
    angle = torch.arange(positions, device="cuda")[:, None] * 10000.0 ** (-torch.arange(max(rot // 2, 1), device="cuda") / max(rot // 2, 1))
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float() if rot else None
    if layout == "pairs":  # keys and values side by side, tokens before heads
        pool = torch.full((20, 2, P, H, D), 7.0, dtype=dt, device="cuda")
        key, value = pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2)
    else:
        pool = torch.full((2, 20, H, P, D), 7.0, dtype=dt, device="cuda")
        key, value = pool[0], pool[1]
    slots = torch.randperm(20 * P, generator=torch.Generator().manual_seed(3))[: B * T].reshape(B, T)
    slots[1, 2:] = -1  # a request with two new tokens
    position = torch.randint(0, positions, (B, T), generator=torch.Generator().manual_seed(4)).to(torch.int32)
    position[0, 0], position[2, 3] = 0, positions - 1
    plan = rheo.CachePlan(cfg, slot=slots.cuda(), position=position.cuda())
    ws = rheo.CacheWorkspace(cfg)
    q0, k0, v0 = q.clone(), k.clone(), v.clone()
    out = q if layout == "in place" else torch.full((B, T, Hq, D), 9.0, dtype=dt, device="cuda")
    rheo.qk_norm_rope(cfg, q, k, v, qw, kw, cos_sin, plan, key, value, out, ws, eps=1e-5, interleaved=interleaved)
    assert rheo.scratch_status(ws) == 0
    seen = torch.zeros((20, P), dtype=torch.bool)
    for b in range(B):
        for t in range(T):
            s = int(slots[b, t])
            if s < 0:
                assert not out[b, t].any()
                continue
            page, row = s // P, s % P
            seen[page, row] = True
            for x, w, got in ((q0[b, t], qw, out[b, t]), (k0[b, t], kw, key[page, :, row])):
                want = ref.rope(x, w, 1e-5, cos_sin, int(position[b, t]), rot, interleaved)
                # a dozen roundings of terms no larger than the pair's two; sum of squares: D of them, halved by the root
                big = ref.rope(x, w, 1e-5, None, 0, 0, False).abs().amax(-1, keepdim=True)
                tol = (D + 24) * ref.U * 2 * big + (2.0 ** -8 * want.abs() * 1.01 if dtype == "bf16" else 0)
                assert ((got.double() - want).abs() <= tol).all()
            assert torch.equal(value[page, :, row], v0[b, t])
    rest = ~seen.cuda()
    assert (key.transpose(1, 2)[rest] == 7).all() and (value.transpose(1, 2)[rest] == 7).all()


def test_norm_rope_flags_bad_slots_and_positions():
    cfg = _cfg(batch=1, tokens=4, pages=2)
    x = torch.ones((1, 4, 8, 64), device="cuda")
    q, k, v = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]
    cs = torch.ones((10, 64), device="cuda")
    key, value = (y[0] for y in rheo.make_cache(cfg))
    plan = rheo.CachePlan(cfg, slot=torch.tensor([[0, 32, 1, 2]], device="cuda"), position=_i32([[0, 1, 10, -1]]))
    ws, out = rheo.CacheWorkspace(cfg), torch.full((1, 4, 4, 64), 5.0, device="cuda")
    rheo.qk_norm_rope(cfg, q, k, v, None, None, cs, plan, key, value, out, ws)
    assert rheo.scratch_status(ws) == rheo.STATUS_BAD_INDEX
    assert out[0, 0].any() and not out[0, 1:].any()
    assert key[0, :, 0].any() and not key[0, :, 1:].any() and not key[1].any()


def test_norm_rope_past_32_bits_of_elements():
    """A pool of more than 2^32 elements: the last page's lines are stored and read at their own places."""
    cfg = _cfg(batch=1, tokens=2, pages=2 ** 18 + 3, page_size=128, max_pages=4, q_heads=2, kv_heads=2, head_dim=64, dtype="bf16")
    pool = torch.zeros((cfg.pages, 2, 128, 64), dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, 2, 6, 64), generator=g, device="cuda").to(torch.bfloat16)
    table = torch.tensor([[cfg.pages - 1, 0, 0, 0]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([[(cfg.pages - 1) * 128, (cfg.pages - 1) * 128 + 1]], device="cuda")
    plan = rheo.CachePlan(cfg, slot=slots, position=_i32([[0, 1]]))
    ws, out = rheo.CacheWorkspace(cfg), torch.empty((1, 2, 2, 64), dtype=torch.bfloat16, device="cuda")
    key, value = pool, torch.zeros_like(pool)
    rheo.qk_norm_rope(cfg, x[:, :, :2], x[:, :, 2:4], x[:, :, 4:], None, None, None, plan, key, value, out, ws)
    assert torch.equal(key[-1, :, :2].transpose(0, 1), x[0, :, 2:4]) and not key[:-1].any()
    got = torch.empty_like(out)
    rheo.tree_attend(cfg, out, key, value, rheo.Pages(cfg, block_table=table), _i32([0]), got, ws)
    o, lse, A, S = ref.attend(out, key, value, table, [0], [2], None, 64 ** -0.5)
    e, _ = ref.attend_bounds(o, lse, A, S, 64, 2, True)
    assert ((got.double() - o).abs() <= e).all()
    assert rheo.scratch_status(ws) == 0


# ---------------------------------------------------------------- commit

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,layers,layout", [(64, 1, 1, "heads"), (128, 8, 3, "tokens"), (64, 3, 5, "pairs"), (128, 2, 2, "heads")])
def test_commit_moves_the_path(dtype, D, H, layers, layout):
    T, P, depth = 40, 16, 12
    ctx = [0, 15, 16, 33, 7, 100, 64]
    paths = [[], [1], [3], [1, 2, 5], list(range(1, 13)), [2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13],
             [3, 5, 7, 9, 11, 13, 15, 17, 19, 39]]
    B = len(ctx)
    cfg = _cfg(batch=B, tokens=T, pages=60, page_size=P, max_pages=10, kv_heads=H, q_heads=H, head_dim=D, dtype=dtype)
    g = torch.Generator().manual_seed(D + H)
    table = _tables(cfg, [c + T for c in ctx], g)
    x = torch.randn((2, layers, 60, H, P, D), generator=g).to(cfg.torch_dtype).cuda()
    if layout == "tokens":
        key, value = (y.transpose(2, 3).contiguous().transpose(2, 3) for y in x)
    elif layout == "pairs":
        both = x.permute(1, 2, 0, 3, 4, 5).contiguous()
        key, value = both[:, :, 0], both[:, :, 1]
    else:
        key, value = x[0], x[1]
    want_k, want_v = key.clone(), value.clone()
    for b, path in enumerate(paths):
        for k, node in enumerate(path):
            (p0, r0), (p1, r1) = (ref.place(table[b], ctx[b] + y, P) for y in (node, k + 1))
            want_k[:, p1, :, r1] = want_k[:, p0, :, r0].clone()
            want_v[:, p1, :, r1] = want_v[:, p0, :, r0].clone()
    nodes = [p + [-1] * (depth - len(p)) for p in paths]
    ws, nxt = rheo.CacheWorkspace(cfg), torch.full((B,), -5, dtype=torch.int32, device="cuda")
    rheo.cache_commit(cfg, key, value, rheo.Pages(cfg, block_table=table), _i32(ctx), _i32([len(p) for p in paths]),
                      _i32(nodes), nxt, ws)
    assert rheo.scratch_status(ws) == 0
    assert torch.equal(key, want_k) and torch.equal(value, want_v)
    assert nxt.tolist() == [c + 1 + len(p) for c, p in zip(ctx, paths)]


def test_commit_flags_broken_paths_and_leaves_them():
    cfg = _cfg(batch=7, tokens=9, pages=40, max_pages=4)
    ctx = [10, 10, 10, 10, 10, -3, 60]
    nodes = [[2, 2, -1], [3, 1, -1], [9, -1, -1], [1, 2, 3], [4, 5, 6], [2, 3, -1], [4, -1, -1]]
    n = [2, 2, 1, 4, 3, 2, 1]
    g = torch.Generator().manual_seed(1)
    table = _tables(cfg, [64] * 7, g) if cfg.pages >= 28 else None
    key, value = rheo.make_cache(cfg)
    key.copy_(torch.randn(key.shape, generator=g))
    value.copy_(torch.randn(key.shape, generator=g))
    k0, v0 = key.clone(), value.clone()
    ws, nxt = rheo.CacheWorkspace(cfg), torch.zeros(7, dtype=torch.int32, device="cuda")
    rheo.cache_commit(cfg, key, value, rheo.Pages(cfg, block_table=table), _i32(ctx), _i32(n), _i32(nodes), nxt, ws)
    assert rheo.scratch_status(ws) == rheo.STATUS_BAD_INDEX | rheo.STATUS_BAD_LENGTH
    for k, node in enumerate(nodes[4]):
        (p0, r0), (p1, r1) = (ref.place(table[4], 10 + y, 16) for y in (node, k + 1))
        k0[:, p1, :, r1], v0[:, p1, :, r1] = k0[:, p0, :, r0].clone(), v0[:, p0, :, r0].clone()
    assert torch.equal(key, k0) and torch.equal(value, v0)
    assert nxt.tolist() == [10, 10, 10, 10, 14, -3, 60]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_of_dimensions_of_one_do_not_count(dtype):
    """One request, one token, one head: torch may give these dimensions any stride."""
    cfg = _cfg(batch=1, tokens=1, pages=2, max_pages=2, q_heads=1, kv_heads=1, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    dt, D = cfg.torch_dtype, cfg.head_dim
    odd = lambda: torch.randn(D, generator=g, device="cuda").to(dt).as_strided((1, 1, 1, D), (7, 5, 3, 1))  # noqa: E731
    q, k, v = odd(), odd(), odd()
    key, value = rheo.make_cache(cfg, 1)
    pages, plan, ws = rheo.Pages(cfg), rheo.CachePlan(cfg), rheo.CacheWorkspace(cfg)
    rheo.cache_reserve(cfg, _i32([0]), pages, plan, ws)
    q_out, out = torch.zeros((1, 1, 1, D), dtype=dt, device="cuda"), torch.zeros(D, dtype=dt, device="cuda")
    rheo.qk_norm_rope(cfg, q, k, v, None, None, None, plan, key[0], value[0], q_out, ws)
    rheo.tree_attend(cfg, q, key[0], value[0], pages, _i32([0]), out.as_strided((1, 1, 1, D), (9, 9, 9, 1)), ws)
    assert rheo.scratch_status(ws) == 0
    assert torch.equal(q_out.flatten(), q.flatten()) and torch.equal(out, v.flatten())
