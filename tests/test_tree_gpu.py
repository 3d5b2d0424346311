"""Attention of trees of drafted tokens over the paged cache against a plain implementation in 64 bits: types, kinds, head layouts,
masks of one word and of several, masks that hide everything, masks at page and tile borders, bad pages and lengths."""
import math

import pytest
import torch

import serving_ref as R
import tree_ref as T
from test_paged_gpu import Cache, check_attention, fn

pytestmark = pytest.mark.gpu


def attend(M, c, G, sets, n_words=None, max_q=None, q=None, fill=-1):
    """sets[b][i]: what token i of sequence b sees among the new ones, as an integer of bits."""
    q = c.rows(c.H_kv * G) if q is None else q
    scale = 1 / math.sqrt(c.D)
    n_words = n_words or max(1, -(-max(len(s) for s in sets) // 64))
    mask = T.mask_tensor(c.T, c.start, sets, n_words, fill)
    args, scales = c.on_gpu()
    o = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    ws = torch.full((M.attn_paged_tree_workspace_bytes(c.T, len(c.kv_len), q.shape[1], c.H_kv, c.D) // 4,), float("nan"), device="cuda")
    got = fn(M, "attn_paged_tree", c.dt)(q.cuda(), *args, mask.cuda(), **scales, o=o, lse=lse, workspace=ws, max_q=max_q)
    assert got[0] is o and got[1] is lse
    torch.cuda.synchronize()
    return q, o.cpu(), lse.cpu(), T.attention(q.double(), *c.values(), c.table, c.start, c.kv_len, mask, scale)


def trees(news, seed):
    return [T.random_tree(n, seed + b) for b, n in enumerate(news)]


SHAPES = [  # news, kvs, H_kv, G, D, page
    ([1], [1], 1, 1, 64, 16),
    ([7], [1000], 3, 1, 64, 16),
    ([4] * 5, [17, 4, 300, 64, 129], 2, 4, 128, 16),
    ([15, 1, 3], [2300, 70, 3], 1, 8, 128, 256),
    ([6], [700], 2, 5, 256, 32),
    ([2], [33], 1, 40, 128, 64),                          # 40 query heads on one key head
    ([3, 0, 1, 31], [90, 50, 1, 1030], 2, 4, 256, 16),
    ([33, 1], [333, 6], 2, 3, 64, 128),                   # 99 rows
    ([64, 2], [64, 500], 2, 4, 128, 16),                  # nothing in front of a tree
    ([130, 1, 65], [500, 777, 77], 1, 2, 64, 64),         # masks of three words
    ([65], [1200], 2, 1, 256, 128),
    ([77], [2500], 1, 8, 256, 32),
    ([200], [4500], 1, 4, 128, 32),
    ([63, 64, 5], [1063, 96, 4000], 1, 8, 128, 16),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n%s_kv%s_H%d_G%d_D%d_p%d" % (max(s[0]), max(s[1]), *s[2:]))
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
def test_trees_match_the_formula(shape, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    news, kvs, H, G, D, page = shape
    c = Cache(news, kvs, H, D, page, dt, e4m3, 41, front=2, behind=3)
    q, o, lse, ref = attend(M, c, G, trees(news, 5), max_q=max(news))
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n, G", [(5, 2), (40, 8)])
def test_masks_of_every_kind(D, e4m3, n, G):
    """Nothing, only others, everything (bits behind the last token too), the first and the last word of several."""
    from paper_2512_18134_amd import binding as M
    kvs = [n, n + 1, 10 * n + 3, 700]
    sets = [[0] * n, [((1 << n) - 1) ^ 1 << i for i in range(n)], [(1 << 192) - 1] * n, [1 << n - 1 | 1 << 191] * n]
    c = Cache([n] * 4, kvs, 2, D, 16, "bf16", e4m3, 43)
    q, o, lse, ref = attend(M, c, G, sets, n_words=3, max_q=n)
    check_attention(c, o, lse, ref)
    assert (o[:n] == 0).all() and (lse[:n] == -math.inf).all()           # nothing in front of the first tree either


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D, n, G", [(64, 9, 4), (128, 70, 4), (256, 70, 2)])
def test_a_triangle_is_the_causal_mask(D, n, G, e4m3):
    """The same rows by the same kernels (or others: the same formula) as attn_paged_fwd."""
    from paper_2512_18134_amd import binding as M
    c = Cache([n, n - 1], [900, n - 1], 2, D, 32, "bf16", e4m3, 47)
    sets = [T.lower_triangle(n), T.lower_triangle(n - 1)]
    q, o, lse, ref = attend(M, c, G, sets, max_q=n)
    check_attention(c, o, lse, ref)
    args, scales = c.on_gpu()
    want, want_lse = M.attn_paged_fwd(q.cuda(), *args, **scales, max_q=n)
    check_attention(c, want.cpu(), want_lse.cpu(), ref)


@pytest.mark.parametrize("D, n, G", [(128, 3, 4), (128, 50, 8), (256, 50, 4), (64, 50, 8)])
def test_new_tokens_behind_the_mask_are_seen_by_none(D, n, G):
    from paper_2512_18134_amd import binding as M
    c = Cache([n, 100], [400, 300], 2, D, 16, "bf16", False, 53)
    sets = [[(1 << n) - 1] * n, [(1 << 64) - 1] * 100]
    q, o, lse, ref = attend(M, c, G, sets, n_words=1, max_q=100)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D, G", [(64, 2), (128, 8), (256, 4)])
def test_pages_and_lengths_that_are_wrong_stay_in_bounds(D, G, e4m3):
    """Missing pages in front of a tree and inside it, page numbers beyond the pool, a length beyond the table, one below the number
    of new tokens, a negative one."""
    from paper_2512_18134_amd import binding as M
    n = 40
    c = Cache([n] * 5, [400, 300, 200, 150, 100], 2, D, 16, "bf16", e4m3, 59)
    c.table[0, 3] = -1
    c.table[0, 23] = c.n_pages                             # positions 368 .. 383 of 400: inside the tree
    c.table[1, :] = -7
    c.kv_len[2] = 10 ** 9
    c.table[2, -(-200 // 16):] = -1
    c.kv_len[3] = 25
    c.kv_len[4] = -3
    for i in range(2):                                     # (a place that is seen now may hold anything but NaN)
        if e4m3:
            c.pages[i].view(torch.uint8)[c.pages[i].view(torch.uint8) == 0x7f] = 0x11
            c.scale[i][c.scale[i] == 255] = 120
        else:
            c.pages[i][torch.isnan(c.pages[i])] = 1.0
    q, o, lse, ref = attend(M, c, G, trees([n] * 5, 7), max_q=n)
    check_attention(c, o, lse, ref)


def test_rows_of_a_batch_of_both_kinds_of_kernels_and_many_sequences():
    from paper_2512_18134_amd import binding as M
    news = [1 + (7 * b) % 5 for b in range(150)]
    news[17], news[91] = 90, 70
    kvs = [n + (37 * b) % 300 for b, n in enumerate(news)]
    c = Cache(news, kvs, 1, 128, 16, "bf16", False, 61, front=1, behind=5)
    q, o, lse, ref = attend(M, c, 4, trees(news, 9), max_q=90)
    check_attention(c, o, lse, ref)
    q, o2, lse2, ref = attend(M, c, 4, trees(news, 9), max_q=1, q=q)       # a wrong bound costs speed alone
    check_attention(c, o2, lse2, ref)


def test_strided_queries_and_a_given_stream():
    from paper_2512_18134_amd import binding as M
    c = Cache([20, 9], [500, 77], 2, 128, 16, "bf16", False, 67)
    fused = torch.randn((c.T, 12, 128), generator=c.gen).bfloat16()
    sets = trees([20, 9], 11)
    q, o, lse, ref = attend(M, c, 4, sets, q=fused[:, :8].contiguous())
    check_attention(c, o, lse, ref)
    args, _ = c.on_gpu()
    mask = T.mask_tensor(c.T, c.start, sets, 1).cuda()
    dev, side = fused.cuda(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = M.attn_paged_tree(dev[:, :8], *args, mask, max_q=20, stream=side)
    side.synchronize()
    assert torch.equal(got[0].cpu(), o) and torch.equal(got[1].cpu(), lse)


def test_long_sequences_are_cut_and_joined_and_repeat_bit_for_bit():
    from paper_2512_18134_amd import binding as M
    for n, G in ((3, 4), (64, 8)):
        c = Cache([n, 1], [9000, 30], 1, 128, 64, "bf16", False, 71)
        q, o, lse, ref = attend(M, c, G, trees([n, 1], 13), max_q=n)
        check_attention(c, o, lse, ref)
        for _ in range(3):
            q, o2, lse2, _ = attend(M, c, G, trees([n, 1], 13), max_q=n, q=q)
            assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D, e4m3", [(64, False), (128, False), (128, True), (256, True)])
def test_ranges_of_keys_of_which_a_row_sees_none(D, e4m3):
    """A tree longer than the ranges that the walk is cut into: most rows see nothing of the last ones, and the first rows, without pages in front of
    them, of all but one."""
    from paper_2512_18134_amd import binding as M
    n = 600
    c = Cache([n], [6000], 1, D, 16, "bf16", e4m3, 73)
    sets = T.random_tree(n, 21)
    sets[7], sets[599] = 0, 1 << 599
    q, o, lse, ref = attend(M, c, 1, [sets], max_q=n)
    check_attention(c, o, lse, ref)
    for missing in ((6000 - n) // 16, (6000 - n) // 16 + 1):    # of what lies before, eight positions are left, then none
        c.table[0, :missing] = -1
        del c._gpu
        q, o, lse, ref = attend(M, c, 1, [sets], max_q=n, q=q)
        check_attention(c, o, lse, ref)
    assert lse[7, 0] == -math.inf and (o[7] == 0).all() and torch.isfinite(lse[599]).all()
