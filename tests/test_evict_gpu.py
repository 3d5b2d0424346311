"""Which places of the cache are kept, and the moves, against plain implementations: whole numbers, so equal ones."""
import math

import pytest
import torch

import evict_ref as E
from test_paged_gpu import Cache

pytestmark = pytest.mark.gpu


def run_select(M, weights, kv_len, keep, moves, stamps=None, seen=None, **kw):
    on = lambda t: None if t is None else t.cuda()
    dst, src, new_len = M.attn_cache_select(weights.cuda(), kv_len.cuda(), keep.cuda(), moves, on(stamps), on(seen), **kw)
    torch.cuda.synchronize()
    got = [t.cpu() for t in (dst, src, new_len)]
    for g, w in zip(got, E.select(weights, kv_len, keep, moves, stamps, seen, **kw)):
        assert torch.equal(g, w)
    return got


i32 = lambda x: torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("kind", ["spread", "few", "zeros", "special"])
@pytest.mark.parametrize("width, kvs, keeps", [
    (16, [1, 2, 16, 0], [1, 1, 5, 3]), (64, [64, 63, 33, 40], [0, 62, -4, 40]), (160, [160, 129, 64, 65], [7, 128, 63, 1]),
    (2048, [2048, 2047, 1500, 1025], [1024, 2046, 1, 512]), (5008, [5000, 4097, 3333, 100], [4999, 2000, 1111, 200])])
def test_select_matches_a_sort(width, kvs, keeps, kind):
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(width)
    w = torch.randn((4, 3, width), generator=gen).mul(2).exp() * 1e-3
    if kind == "few":
        w = torch.randint(0, 3, w.shape, generator=gen).float()          # ties everywhere
    elif kind == "zeros":
        w = torch.where(torch.rand(w.shape, generator=gen) < 0.9, torch.zeros(()), w) * torch.where(torch.rand(w.shape, generator=gen) < 0.5, -0.0, 1.0).sign()
        w[:, 1] = -0.0
    elif kind == "special":
        for x in (math.inf, -math.inf, math.nan, -math.nan, 1e-42, -1e-42, -1.0):
            w[torch.rand(w.shape, generator=gen) < 0.1] = x
    moves = max(1, max(min(max(k, 0), kv - max(k, 0)) for k, kv in zip(keeps, kvs)))
    run_select(M, w, i32(kvs), i32(keeps), moves)
    run_select(M, w, i32(kvs), i32(keeps), moves + 5, sinks=2, recent=3)
    run_select(M, w, i32(kvs), i32(keeps), moves, sinks=0, recent=10 ** 6)      # all of them always stay: the lowest places


def test_select_by_stamps():
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(5)
    B, H, width = 3, 2, 512
    w = torch.rand((B, H, width), generator=gen)
    stamps = torch.stack([torch.randperm(700, generator=gen)[:width] for _ in range(B * H)]).view(B, H, width).to(torch.int32)
    for sinks, recent in ((0, 0), (4, 0), (0, 50), (16, 128), (300, 300), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1)):
        run_select(M, w, i32([512, 400, 17]), i32([256, 100, 3]), 256, stamps, i32([700, 650, 10]), sinks=sinks, recent=recent)
    run_select(M, w, i32([512, 400, 17]), i32([256, 100, 3]), 256, stamps, i32([-5, 2 ** 31 - 1, 0]), sinks=2, recent=9)


def test_a_sequence_with_more_moves_than_the_lists_hold_drops_nothing():
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(6)
    w = torch.rand((4, 2, 256), generator=gen)
    dst, src, new_len = run_select(M, w, i32([256, 200, 180, 10 ** 9]), i32([100, 195, 10, 240]), 10)
    assert new_len.tolist() == [256, 195, 10, 256]
    run_select(M, w, i32([-4, 200, 180, 10 ** 9]), i32([100, 195, 10, 240]), 16)


def test_select_of_long_sequences():
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(7)
    w = torch.randn((2, 2, 131072), generator=gen).mul(2).exp()
    w[1] = torch.randint(0, 50, w[1].shape, generator=gen).float()
    run_select(M, w, i32([131072, 100001]), i32([8192, 65000]), 40000, sinks=4, recent=1000)


@pytest.mark.parametrize("kind", ["spread", "few", "special"])
@pytest.mark.parametrize("width, kvs, keeps", [
    (8208, [8208, 8193, 5000, 8208], [100, 8192, 4999, 8207]), (16384, [16384, 9000, 16383, 12289], [5000, 8999, 16382, 1]), (16400, [16400, 16385, 16384, 20], [8001, 16384, 1, 7]),
    (50000, [50000, 49153, 33000, 50000], [32768, 16383, 16385, 3])])
def test_select_of_lists_in_parts(width, kvs, keeps, kind):
    """Ends at, before and behind the borders of the parts, which begin anew at the new length."""
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(width)
    w = torch.randn((4, 1, width), generator=gen).mul(2).exp() * 1e-3
    if kind == "few":
        w = torch.randint(0, 3, w.shape, generator=gen).float()
    elif kind == "special":
        for x in (math.inf, math.nan, -1.0, 0.0):
            w[torch.rand(w.shape, generator=gen) < 0.2] = x
    moves = max(min(k, kv - k) for k, kv in zip(keeps, kvs))
    run_select(M, w, i32(kvs), i32(keeps), moves, sinks=3, recent=50)
    stamps = torch.stack([torch.randperm(width + 9, generator=gen)[:width] for _ in range(4)]).view(4, 1, width).to(torch.int32)
    run_select(M, w, i32(kvs), i32(keeps), moves // 2, stamps, i32([width + 9] * 4), sinks=100, recent=1000)


def test_select_in_a_given_workspace_that_holds_something_else():
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(8)
    w = torch.rand((2, 2, 20000), generator=gen)
    need = M.attn_cache_select_workspace_bytes(2, 2, 20000)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        got = M.attn_cache_select(w.cuda(), i32([20000, 9000]).cuda(), i32([500, 8000]).cuda(), 1000, workspace=ws)
        for g, want in zip(got, E.select(w, i32([20000, 9000]), i32([500, 8000]), 1000)):
            assert torch.equal(g.cpu(), want)


def dirty(c):
    """Every place holds something of its own."""
    for i in range(2):
        if c.e4m3:
            c.pages[i].view(torch.uint8)[:] = torch.randint(0, 256, c.pages[i].shape, generator=c.gen, dtype=torch.uint8)
            c.scale[i][:] = torch.randint(0, 256, c.scale[i].shape, generator=c.gen, dtype=torch.uint8)
        else:
            c.pages[i].view(torch.int16)[:] = torch.randint(-32768, 32768, c.pages[i].shape, generator=c.gen, dtype=torch.int16)


def run_move(M, c, dst, src, state=True):
    dirty(c)
    B, L = len(c.kv_len), c.table.shape[1] * c.page
    weights = torch.rand((B, c.H_kv, L), generator=c.gen) if state else None
    stamps = torch.randint(0, 10 ** 9, (B, c.H_kv, L), generator=c.gen, dtype=torch.int32) if state else None
    args, scales = c.on_gpu()
    on = lambda t: None if t is None else t.cuda()
    w, st = on(weights), on(stamps)
    M.attn_cache_move(args[0], args[1], args[2], dst.cuda(), src.cuda(), **scales, weights=w, stamps=st)
    torch.cuda.synchronize()
    as_int = lambda t: t.view(torch.uint8 if c.e4m3 else torch.int16)
    tensors = [as_int(p) for p in c.pages] + [s for s in c.scale if s is not None]
    got = [as_int(p.cpu()) for p in args[:2]] + [s.cpu() for s in scales.values() if s is not None]
    rows = [weights, stamps] if state else []
    E.move(tensors, rows, c.table, c.page, dst, src)
    for g, want in zip(got + ([w.cpu(), st.cpu()] if state else []), tensors + rows):
        assert torch.equal(g, want)


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", True)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads", ["all", "each"])
def test_short_lists_may_overlap(D, dt, e4m3, heads):
    """Accepted paths, reversals, cycles: every source is read before anything is written."""
    from paper_2512_18134_amd import binding as M
    c = Cache([1] * 4, [200, 130, 64, 300], 3, D, 16, dt, e4m3, 31)
    H = 1 if heads == "all" else 3
    for moves in (1, 5, 128):
        dst, src = torch.full((4, H, moves), -1, dtype=torch.int32), torch.full((4, H, moves), -1, dtype=torch.int32)
        for b, kv in enumerate([200, 130, 64, 300]):
            for h in range(H):
                n = min(moves, kv, [moves, 3, 7, moves][b])
                places = torch.randperm(kv, generator=c.gen)[:n].to(torch.int32)
                dst[b, h, :n] = places
                src[b, h, :n] = places.roll(1) if b < 2 else places.sort().values if b == 2 else torch.randint(0, kv, (n,), generator=c.gen)
        run_move(M, c, dst, src, state=heads == "each")
        del c._gpu


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_lists_of_select(D, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    kvs, keeps = [1500, 900, 40, 1200], [700, 870, 39, 1100]
    c = Cache([1] * 4, kvs, 2, D, 32, dt, e4m3, 33)
    w = torch.rand((4, 2, c.table.shape[1] * 32), generator=c.gen)
    dst, src, _ = run_select(M, w, i32(kvs), i32(keeps), 777)
    run_move(M, c, dst, src)


@pytest.mark.parametrize("moves", [3, 300])
def test_places_that_are_none_move_nothing(moves):
    from paper_2512_18134_amd import binding as M
    c = Cache([1] * 2, [500, 400], 2, 128, 16, "bf16", False, 35)
    c.table[0, 4], c.table[0, 20], c.table[1, 0] = -1, c.n_pages, 10 ** 9
    L = c.table.shape[1] * 16
    places = torch.stack([torch.stack([torch.randperm(L, generator=c.gen)[:moves] for _ in range(2)]) for _ in range(4)]).view(2, 2, 2, moves)
    dst = places[0].to(torch.int32)
    src = torch.where(places[1] % 3 == 0, -2 ** 31 + places[1], places[1]).to(torch.int32)
    if moves > 128:                                        # disjoint
        dst = torch.where(dst < 256, dst, -1)
        src = torch.where(src >= 256, src, 2 ** 31 - 1)
    dst[:, :, 1], src[:, :, 2] = L, L
    run_move(M, c, dst.contiguous(), src.contiguous())
