"""Trees, weights, choice and moves where offsets pass 32 bits: pools and arrays beside them beyond 2^32 elements, queries far apart, tables wider
than any sequence."""
import math

import pytest
import torch

import evict_ref as E
import serving_ref as R
import tree_ref as T
from test_paged_gpu import check_attention

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.tensor(x, dtype=torch.int32)


class Far:
    """Sequences whose pages lie at the end of a pool of more than 2^32 elements; `small` is a pool of their pages alone."""

    def __init__(self, D, kvs, seed):
        gen = torch.Generator().manual_seed(seed)
        H, page = 8, 256
        self.n_pages = (1 << 32) // (H * page * D) + 40
        self.dt, self.kv_len, self.gen = "bf16", i32(kvs), gen
        need = [-(-kv // page) for kv in kvs]
        ids = torch.randperm(40, generator=gen)[:sum(need)]
        self.table = torch.full((len(kvs), max(need)), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = (self.n_pages - 40 + ids[at:at + n]).to(torch.int32)
            at += n
        self.small_table = torch.where(self.table >= 0, self.table - (self.n_pages - 40), -1)
        self.small = [torch.randn((40, H, page, D), generator=gen).bfloat16() for _ in "kv"]
        self.pages = [torch.empty((self.n_pages, H, page, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        for big, x in zip(self.pages, self.small):
            big[-40:] = x.cuda()


@pytest.mark.parametrize("D", [128, 256])
def test_pools_beyond_two_to_the_32_elements(D):
    from paper_2512_18134_amd import binding as M
    n, kvs = [40, 3], [700, 500]
    f = Far(D, kvs, 3)
    start = i32([0, 40, 43])
    q = torch.randn((43, 16, D), generator=f.gen).bfloat16()
    mask = T.mask_tensor(43, start, [T.random_tree(m, 1) for m in n], 1)
    index = f.table.cuda(), start.cuda(), f.kv_len.cuda()
    values = [x.double() for x in f.small]
    for max_q in (40, 1):
        o, lse = M.attn_paged_tree(q.cuda(), *f.pages, *index, mask.cuda(), max_q=max_q)
        check_attention(f, o.cpu(), lse.cpu(), T.attention(q.double(), *values, f.small_table, start, f.kv_len, mask, 1 / math.sqrt(D)))
    lse = torch.randn((43, 16), generator=f.gen) + 3
    zeros = torch.zeros((2, 8, f.table.shape[1] * 256))
    want, bound, _ = E.weigh(q.double(), lse, values[0], f.small_table, start, f.kv_len, zeros, 1.0, True, 1 / math.sqrt(D))
    for max_q in (40, 1):
        w = M.attn_cache_weigh(q.cuda(), lse.cuda(), f.pages[0], *index, zeros.cuda(), max_q=max_q)
        assert ((w.cpu().double() - want).abs() <= bound + 1e-30).all()
    dst, src = torch.full((2, 8, 200), -1, dtype=torch.int32), torch.full((2, 8, 200), -1, dtype=torch.int32)
    for b in range(2):
        for h in range(8):
            dst[b, h, :150] = torch.randperm(250, generator=f.gen)[:150]
            src[b, h, :150] = 250 + torch.randperm(250, generator=f.gen)[:150]
    M.attn_cache_move(*f.pages, index[0], dst.cuda(), src.cuda())
    E.move([x.view(torch.int16) for x in f.small], [], f.small_table, 256, dst, src)
    for big, x in zip(f.pages, f.small):
        assert torch.equal(big[-40:].cpu().view(torch.int16), x.view(torch.int16))


def test_arrays_beside_the_cache_beyond_two_to_the_32_elements():
    """A table of 2^24 places, of which the sequences have a few hundred: the last sequence's rows lie behind 2^32 elements."""
    from paper_2512_18134_amd import binding as M
    B, H, page, D = 34, 8, 256, 64
    width = 1 << 16
    gen = torch.Generator().manual_seed(5)
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[B - 1, :3] = i32([4, 1, 2])
    pages = [torch.randn((5, H, page, D), generator=gen).bfloat16() for _ in "kv"]
    weights = torch.empty((B, H, width * page), device="cuda")
    stamps = torch.empty((B, H, width * page), dtype=torch.int32, device="cuda")
    assert weights[: B - 1].numel() > 1 << 32
    had = torch.rand((H, 768), generator=gen)
    weights[B - 1, :, :768] = had.cuda()
    kv_len = i32([0] * (B - 1) + [600])
    for n in (2, 100):                                     # both kernels
        start = i32([0] * B + [n])
        q, lse = torch.randn((n, 16, D), generator=gen).bfloat16(), torch.randn((n, 16), generator=gen) + 3
        seen = i32([0] * (B - 1) + [700])
        want, bound, _ = E.weigh(q.double(), lse, pages[0].double(), table[B - 1:, :3], i32([0, n]), kv_len[B - 1:], had[None], 0.5, True, 0.125)
        stamps[B - 1, :, :768] = -1
        weights[B - 1, :, :768] = had.cuda()
        M.attn_cache_weigh(q.cuda(), lse.cuda(), pages[0].cuda(), table.cuda(), start.cuda(), kv_len.cuda(), weights, stamps=stamps,
                           seen=seen.cuda(), decay=0.5, max_q=n)
        got = weights[B - 1, :, :768].cpu().double()
        assert ((got - want[0]).abs() <= bound[0] + 1e-30).all()
        numbers = stamps[B - 1, :, :768].cpu()
        assert (numbers[:, 600 - n:600] == torch.arange(700 - n, 700)).all() and (numbers[:, :600 - n] == -1).all() and (numbers[:, 600:] == -1).all()
    stamps[B - 1, :, :768] = torch.arange(768, dtype=torch.int32, device="cuda")
    keep = i32([0] * (B - 1) + [250])
    small = weights[B - 1:, :, :768].cpu()
    want = E.select(small, kv_len[B - 1:], keep[B - 1:], 300, recent=20)
    dst, src, new_len = M.attn_cache_select(weights, kv_len.cuda(), keep.cuda(), 300, stamps, kv_len.cuda(), recent=20)
    assert torch.equal(dst[B - 1:].cpu(), want[0]) and torch.equal(src[B - 1:].cpu(), want[1])
    assert (dst[: B - 1] == -1).all() and (src[: B - 1] == -1).all() and new_len.tolist() == [0] * (B - 1) + [250]
    k = [x.cuda() for x in pages]
    M.attn_cache_move(*k, table.cuda(), dst, src, weights=weights, stamps=stamps)
    rows = [small, torch.arange(768, dtype=torch.int32).expand(1, H, 768).contiguous()]
    E.move([x.view(torch.int16) for x in pages], rows, table[B - 1:, :3], page, *want[:2])
    assert torch.equal(weights[B - 1, :, :768].cpu(), rows[0][0]) and torch.equal(stamps[B - 1, :, :768].cpu(), rows[1][0])
    assert all(torch.equal(a.cpu().view(torch.int16), b.view(torch.int16)) for a, b in zip(k, pages))


def test_queries_too_far_apart_for_the_tile_kernel():
    """Rows of a call that lie more than 2^32 bytes apart are weighed by the row kernel, the same rows side by side by the other."""
    from paper_2512_18134_amd import binding as M
    n, D = 90, 64
    gen = torch.Generator().manual_seed(7)
    pages = torch.randn((8, 2, 64, D), generator=gen).bfloat16().cuda()
    table, start, kv = i32([[3, 1, 7, 0]]).cuda(), i32([0, n]).cuda(), i32([250]).cuda()
    q, lse = torch.randn((n, 4, D), generator=gen).bfloat16().cuda(), (torch.randn((n, 4), generator=gen) + 3).cuda()
    stride = (1 << 32) // (2 * (n - 1)) // 8 * 8 + 64
    far = torch.empty(stride * (n - 1) + 4 * D, dtype=torch.bfloat16, device="cuda").as_strided((n, 4, D), (stride, D, 1))
    far.copy_(q)
    zeros = torch.zeros((1, 2, 256))
    want, bound, _ = E.weigh(q.cpu().double(), lse.cpu(), pages.cpu().double(), table.cpu(), start.cpu(), kv.cpu(), zeros, 1.0, True, 0.125)
    for x in (q, far):
        w = M.attn_cache_weigh(x, lse, pages, table, start, kv, zeros.cuda())
        assert ((w.cpu().double() - want).abs() <= bound + 1e-30).all()
