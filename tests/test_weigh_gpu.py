"""Accumulated attention weights against a plain implementation in 64 bits: types, kinds, head layouts, ragged batches, masks, rows that see
nothing, bad pages and lengths, in place and beside it."""
import math

import pytest
import torch

import evict_ref as E
import serving_ref as R
from test_paged_gpu import Cache, fn

pytestmark = pytest.mark.gpu


def check(M, c, G, causal=True, decay=0.75, stamps=False, in_place=True, max_q=None, empty=(), q=None, repeat=None):
    gen = torch.Generator().manual_seed(91)
    H_q, L = c.H_kv * G, c.table.shape[1] * c.page
    q = c.rows(H_q) if q is None else q
    scale = 1 / math.sqrt(c.D)
    B = len(c.kv_len)
    ref_lse = R.attention(q.double(), c.values()[0], c.values()[0].nan_to_num(), c.table, c.start, c.kv_len, causal, scale)[1]
    lse = ref_lse.float()
    for t in empty:
        lse[t] = -math.inf
    weights = torch.rand((B, c.H_kv, L), generator=gen)
    for b in range(B):                                     # what must not be read
        weights[b, :, max(0, min(int(c.kv_len[b]), L)):] = float("nan")
        n = int(c.start[b + 1] - c.start[b])
        if decay == 0:
            weights[b] = float("nan")
        elif n > 0:
            weights[b, :, max(0, int(c.kv_len[b]) - n):max(0, int(c.kv_len[b]))] = float("nan")
    st = torch.randint(0, 99, (B, c.H_kv, L), generator=gen, dtype=torch.int32) if stamps else None
    seen = (c.kv_len + 17).to(torch.int32) if stamps else None
    want, bound, want_st = E.weigh(q.double(), lse, c.values()[0], c.table, c.start, c.kv_len, weights, decay, causal, scale, st, seen)
    args, scales = c.on_gpu()
    on = lambda t: None if t is None else t.cuda()
    w_in, st_dev = on(weights), on(st)
    out = w_in if in_place else on(weights)
    got = fn(M, "attn_cache_weigh", c.dt)(q.cuda(), lse.cuda(), args[0], *args[2:], w_in, k_scale=scales["k_scale"],
                                          out=None if in_place else out, stamps=st_dev, seen=on(seen), decay=decay, causal=causal,
                                          max_q=max_q)
    assert got is out
    torch.cuda.synchronize()
    y = out.cpu()
    written = torch.zeros(want.shape, dtype=torch.bool)
    for b in range(B):
        if int(c.start[b + 1] - c.start[b]) > 0:
            written[b, :, :max(0, min(int(c.kv_len[b]), L))] = True
    assert torch.equal(y[~written].view(torch.int32), weights[~written].view(torch.int32)), "places of nobody were written"
    err = (y.double() - want).abs()[written]
    assert (err <= bound[written] + 1e-30).all(), float((err - bound[written]).max())
    if stamps:
        assert torch.equal(st_dev.cpu(), want_st)
    if not in_place:
        assert torch.equal(w_in.cpu().view(torch.int32), weights.view(torch.int32))
    return q, y


SHAPES = [  # news, kvs, H_kv, G, D, page
    ([1], [1], 1, 1, 64, 16),
    ([1], [1000], 3, 1, 64, 16),
    ([1] * 5, [17, 1, 300, 64, 129], 2, 4, 128, 16),
    ([1, 1], [2300, 70], 1, 8, 128, 256),
    ([1], [700], 2, 5, 256, 32),
    ([1], [33], 1, 40, 128, 64),
    ([4] * 3, [400, 4, 131], 2, 3, 128, 32),
    ([3, 0, 1, 7], [90, 50, 1, 1030], 2, 4, 256, 16),
    ([5, 1], [5, 6], 2, 16, 64, 128),
    ([100], [100], 2, 4, 128, 16),
    ([130, 1, 37], [500, 777, 37], 1, 2, 64, 64),
    ([65], [1200], 2, 1, 256, 128),
    ([300], [2500], 1, 4, 128, 32),
    ([70, 400], [90, 411], 1, 5, 256, 16),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n%s_kv%s_H%d_G%d_D%d_p%d" % (max(s[0]), max(s[1]), *s[2:]))
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
def test_weights_match_the_formula(shape, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    news, kvs, H, G, D, page = shape
    c = Cache(news, kvs, H, D, page, dt, e4m3, 81, front=2, behind=3)
    q, _ = check(M, c, G, True, 0.75, stamps=True, max_q=max(news))
    check(M, c, G, False, 0.0, in_place=False, q=q)


@pytest.mark.parametrize("decay", [0.0, 1.0, 2.5])
@pytest.mark.parametrize("in_place", [False, True])
def test_decay_and_rows_that_see_nothing(decay, in_place):
    from paper_2512_18134_amd import binding as M
    c = Cache([6, 1, 90], [60, 20, 300], 2, 128, 16, "bf16", False, 83)
    check(M, c, 4, True, decay, in_place=in_place, empty=[0, 5, 6, 50], stamps=True)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D, n", [(64, 3), (128, 150), (256, 3)])
def test_pages_and_lengths_that_are_wrong_stay_in_bounds(D, n, e4m3):
    from paper_2512_18134_amd import binding as M
    c = Cache([n] * 5, [400, 300, 200, 150, 160], 2, D, 16, "bf16", e4m3, 89)
    c.table[0, 3] = -1
    c.table[0, 23] = c.n_pages
    c.table[1, :] = -7
    c.kv_len[2] = 10 ** 9
    c.table[2, -(-200 // 16):] = -1
    c.kv_len[3] = 2
    c.kv_len[4] = -3
    for i in range(2):
        if e4m3:
            c.pages[i].view(torch.uint8)[c.pages[i].view(torch.uint8) == 0x7f] = 0x11
            c.scale[i][c.scale[i] == 255] = 120
        else:
            c.pages[i][torch.isnan(c.pages[i])] = 1.0
    check(M, c, 3, True, 0.5, stamps=True)


def test_a_batch_of_many_sequences_and_long_ones():
    from paper_2512_18134_amd import binding as M
    news = [(7 * b) % 4 for b in range(150)]
    kvs = [n + (37 * b) % 300 for b, n in enumerate(news)]
    c = Cache(news, kvs, 1, 64, 16, "bf16", False, 97, front=1, behind=5)
    check(M, c, 4)
    c = Cache([2, 500], [9000, 4000], 2, 128, 64, "f16", False, 101)
    q, y = check(M, c, 2)
    for _ in range(3):
        assert torch.equal(check(M, c, 2, q=q)[1].nan_to_num(7.0), y.nan_to_num(7.0))


def test_weights_of_a_row_add_up_to_one():
    """What attn_paged_fwd leaves as lse makes the weights of every row and head a distribution."""
    from paper_2512_18134_amd import binding as M
    c = Cache([20, 1], [3000, 77], 2, 128, 32, "bf16", False, 103)
    args, _ = c.on_gpu()
    q = c.rows(8).cuda()
    o, lse = M.attn_paged_fwd(q, *args, max_q=20)
    w = torch.zeros((2, 2, c.table.shape[1] * 32), device="cuda")
    M.attn_cache_weigh(q, lse, args[0], *args[2:], w, max_q=20)
    total = w.double().sum(-1).cpu()
    assert ((total - torch.tensor([[80.0, 80.0], [4.0, 4.0]])).abs() < 1e-4 * total).all()


@pytest.mark.parametrize("D, kv, e4m3", [(64, 16500, False), (128, 16500, True), (128, 16500, False), (256, 8400, False)])
def test_many_rows_on_many_blocks_of_keys(D, kv, e4m3):
    """So many blocks that a wave has keys of its own (with fewer, a workgroup's waves share theirs)."""
    from paper_2512_18134_amd import binding as M
    c = Cache([70, 3], [kv, 200], 8, D, 64, "bf16", e4m3, 107)
    check(M, c, 1, True, 0.5, stamps=True, max_q=70)
    c = Cache([140], [kv], 8, D, 64, "f16", e4m3, 109)
    check(M, c, 1, False, 0.0, in_place=False, empty=[1, 139])


def test_strided_queries():
    from paper_2512_18134_amd import binding as M
    for n, G in ((3, 4), (90, 3)):
        c = Cache([n, 1], [300, 40], 2, 128, 16, "bf16", False, 113)
        fused = torch.randn((c.T, 2 * G + 5, 128), generator=c.gen).bfloat16()
        args, _ = c.on_gpu()
        lse = torch.randn((c.T, 2 * G), generator=c.gen).cuda()
        w = [torch.zeros((2, 2, c.table.shape[1] * 16), device="cuda") for _ in range(2)]
        M.attn_cache_weigh(fused.cuda()[:, 2:2 + 2 * G], lse, args[0], *args[2:], w[0], max_q=n)
        M.attn_cache_weigh(fused[:, 2:2 + 2 * G].contiguous().cuda(), lse, args[0], *args[2:], w[1], max_q=n)
        assert torch.equal(*w) and float(w[0].sum()) > 0
