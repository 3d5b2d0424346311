"""Calls of trees, weights and moves that their headers allow and that stand beside the ordinary ones: more query heads to a key head than a tile has
rows, heads farther apart than rows, weights that are not there yet, one long list for all heads, arrays beside the cache one at a time."""
import pytest
import torch

import evict_ref as E
import tree_ref as T
from test_evict_gpu import dirty
from test_paged_gpu import Cache, check_attention, fn
from test_tree_gpu import attend, trees
from test_weigh_gpu import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D, G, e4m3", [(64, 160, False), (64, 96, True), (128, 160, True), (128, 129, False), (256, 72, False), (256, 65, True)])
def test_more_heads_than_a_tile_has_rows(D, G, e4m3):
    from paper_2512_18134_amd import binding as M
    c = Cache([1, 3], [900, 40], 1, D, 16, "bf16", e4m3, 121)
    check(M, c, G, True, 0.5, stamps=True, max_q=3)
    check(M, c, G, False, 1.0, max_q=1)
    q, o, lse, ref = attend(M, c, G, trees([1, 3], 3), max_q=3)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("D, e4m3", [(64, False), (128, False), (128, True), (256, True)])
def test_a_token_of_several_tiles_in_a_cut_sequence(D, e4m3):
    """40 heads on a key head, taken 16 rows at a time over ranges that are merged."""
    from paper_2512_18134_amd import binding as M
    c = Cache([2, 1], [3000, 17], 1, D, 16, "bf16", e4m3, 127)
    for max_q in (2, 1):
        q, o, lse, ref = attend(M, c, 40, trees([2, 1], 3), max_q=max_q)
        check_attention(c, o, lse, ref)


@pytest.mark.parametrize("n", [3, 90])
@pytest.mark.parametrize("D, dt", [(64, "f16"), (128, "bf16"), (256, "bf16")])
def test_queries_that_lie_head_by_head(n, D, dt):
    """[H_q, T, D] seen as [T, H_q, D], with a gap behind every head."""
    from paper_2512_18134_amd import binding as M
    c = Cache([n, 2], [500, 40], 2, D, 32, dt, False, 131)
    q, o, lse, ref = attend(M, c, 3, trees([n, 2], 7), max_q=n)
    far = torch.full((6, c.T + 5, D), float("nan"), dtype=q.dtype, device="cuda")
    far[:, :c.T] = q.transpose(0, 1).cuda()
    far = far[:, :c.T].transpose(0, 1)
    args, _ = c.on_gpu()
    mask = T.mask_tensor(c.T, c.start, trees([n, 2], 7), max(1, -(-n // 64))).cuda()
    got = fn(M, "attn_paged_tree", dt)(far, *args, mask, max_q=n)
    assert torch.equal(got[0].cpu(), o) and torch.equal(got[1].cpu(), lse)
    w = [torch.zeros((2, 2, c.table.shape[1] * 32), device="cuda") for _ in range(2)]
    for x, rows in zip(w, (q.cuda(), far)):
        fn(M, "attn_cache_weigh", dt)(rows, got[1], args[0], *args[2:], x, max_q=n)
    assert torch.equal(*w) and float(w[0].sum()) > 0


@pytest.mark.parametrize("n", [2, 100])
def test_weights_that_are_not_there_yet(n):
    """weights None: as many as zeros leave, whatever decay says, and nothing is read."""
    from paper_2512_18134_amd import binding as M
    c = Cache([n, 1], [700, 33], 2, 128, 16, "bf16", False, 137)
    args, _ = c.on_gpu()
    q, lse = c.rows(8).cuda(), (torch.randn((c.T, 8), generator=c.gen) + 4).cuda()
    shape = (2, 2, c.table.shape[1] * 16)
    outs = []
    for decay in (0.0, 1.0, 0.5):
        out = torch.full(shape, float("nan"), device="cuda")
        assert M.attn_cache_weigh(q, lse, args[0], *args[2:], None, out=out, decay=decay, max_q=n) is out
        outs.append(out)
    zeros = torch.zeros(shape, device="cuda")
    want = torch.full(shape, float("nan"), device="cuda")
    M.attn_cache_weigh(q, lse, args[0], *args[2:], zeros, out=want, decay=1.0, max_q=n)
    for out in outs:
        assert torch.equal(out.view(torch.int32), want.view(torch.int32))
    for b, kv in enumerate((700, 33)):
        assert torch.isfinite(want[b, :, :kv]).all() and torch.isnan(want[b, :, kv:]).all()


@pytest.mark.parametrize("D, dt, e4m3", [(64, "bf16", False), (128, "bf16", True), (256, "f16", False)])
@pytest.mark.parametrize("beside", ["weights", "stamps", "none"])
def test_one_long_list_for_all_heads(D, dt, e4m3, beside):
    from paper_2512_18134_amd import binding as M
    c = Cache([1] * 3, [1500, 640, 20], 3, D, 16, dt, e4m3, 139)
    dirty(c)
    dst, src = torch.full((3, 1, 333), -1, dtype=torch.int32), torch.full((3, 1, 333), -1, dtype=torch.int32)
    for b, (kv, m) in enumerate(((1500, 333), (640, 300), (20, 9))):
        places = torch.randperm(kv, generator=c.gen)[:2 * m].to(torch.int32)
        dst[b, 0, :m], src[b, 0, :m] = places[:m], places[m:2 * m]
    L = c.table.shape[1] * 16
    weights, stamps = torch.rand((3, 3, L), generator=c.gen), torch.randint(0, 10 ** 9, (3, 3, L), generator=c.gen, dtype=torch.int32)
    given = {"weights": weights} if beside == "weights" else {"stamps": stamps} if beside == "stamps" else {}
    args, scales = c.on_gpu()
    on = {name: t.cuda() for name, t in given.items()}
    M.attn_cache_move(*args[:3], dst.cuda(), src.cuda(), **scales, **on)
    as_int = lambda t: t.view(torch.uint8 if c.e4m3 else torch.int16)
    tensors = [as_int(p) for p in c.pages] + [s for s in c.scale if s is not None]
    E.move(tensors, list(given.values()), c.table, c.page, dst, src)
    for got, want in zip([as_int(p.cpu()) for p in args[:2]] + [s.cpu() for s in scales.values() if s is not None], tensors):
        assert torch.equal(got, want)
    for name, want in given.items():
        assert torch.equal(on[name].cpu(), want)
