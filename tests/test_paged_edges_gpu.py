"""Calls over the paged cache that the entry points allow and are easily forgotten: more query heads to a key head than the row kernel takes, pages
that several sequences share, e4m3 rows of the smallest numbers, hints that are wrong, one long and many empty sequences."""
import math

import pytest
import torch

import serving_ref as R
from test_paged_gpu import Cache, attend, check_attention, fn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", True)])
@pytest.mark.parametrize("D, G", [(64, 130), (64, 300), (128, 200), (256, 65), (256, 129)])
def test_single_tokens_of_many_heads_to_a_key_head(D, G, dt, e4m3):
    """More rows than the row kernel takes in one token: tiles, a batch of them, and tokens among none."""
    from paper_2512_18134_amd import binding as M
    c = Cache([1, 0, 1, 2], [300, 7, 1, 70], 1, D, 16, dt, e4m3, 91, front=1, behind=1)
    for max_q in (2, None):
        _, o, lse, ref = attend(M, c, G, True, max_q)
        check_attention(c, o, lse, ref)


@pytest.mark.parametrize("n", [1, 50])
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True)])
def test_sequences_that_share_pages(n, dt, e4m3):
    """A prefix that three sequences read, a page that stands twice in one sequence."""
    from paper_2512_18134_amd import binding as M
    c = Cache([n, n, n], [260, 260, 200], 2, 128, 16, dt, e4m3, 92)
    c.table[1, :12] = c.table[0, :12]
    c.table[2, :6] = c.table[0, :6]
    c.table[2, 7] = c.table[2, 6]
    _, o, lse, ref = attend(M, c, 4, True, n)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_e4m3_rows_of_the_smallest_numbers(dt):
    """Rows whose amplitude is subnormal in the row type, or only just not."""
    from paper_2512_18134_amd import binding as M
    t, D, n = R.DT[dt], 64, 6
    tiny = torch.finfo(t).smallest_normal
    step = tiny * torch.finfo(t).eps                       # the smallest number
    gen = torch.Generator().manual_seed(93)
    x = torch.zeros(n, 1, D, dtype=torch.float64)
    for r, top in enumerate((step, 3 * step, tiny / 2, tiny - step, tiny, 7 * tiny)):
        x[r, 0] = (torch.rand(D, generator=gen, dtype=torch.float64) * 2 - 1) * top
        x[r, 0, 5] = -top
    x = x.to(t)
    pages = [torch.zeros(1, 1, 16, D).to(torch.float8_e4m3fn).cuda() for _ in "kv"]
    scale = [torch.zeros(1, 1, 16, dtype=torch.uint8, device="cuda") for _ in "kv"]
    index = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([[0]], [0, n], [n])]
    fn(M, "attn_cache_write", dt)(x.cuda(), x.cuda(), *pages, *index, *scale)
    want, e = R.e4m3_row(x)
    assert torch.equal(scale[0].cpu()[0, 0, :n].int() - 127, e[:, 0].int())
    assert torch.equal(R.cached(pages[0].cpu(), scale[0].cpu())[0, :, :n].transpose(0, 1), want)
    k, v = fn(M, "attn_cache_read", dt)(*pages, *index, n, *scale)
    assert torch.equal(k.cpu().double(), want.to(t).double()) and torch.equal(k, v)


@pytest.mark.parametrize("max_q", [1, 2 ** 31 - 1, 2 ** 40])
def test_bounds_on_the_new_tokens_that_are_far_off(max_q):
    from paper_2512_18134_amd import binding as M
    c = Cache([1, 200, 0, 9], [900, 200, 5, 2000], 2, 64, 32, "bf16", False, 94)
    _, o, lse, ref = attend(M, c, 2, True, max_q)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("n, kv", [(1, 5000), (150, 3000)])
@pytest.mark.parametrize("B", [127, 128, 129])
def test_one_sequence_among_empty_ones(B, n, kv):
    """On both sides of the number of sequences from which the cut has a launch of its own."""
    from paper_2512_18134_amd import binding as M
    news, kvs = [0] * B, [0] * B
    news[B - 3], kvs[B - 3] = n, kv
    kvs[4] = 40                                            # a sequence that rests
    c = Cache(news, kvs, 2, 128, 16, "bf16", False, 95, behind=3)
    for max_q in (n, None):
        _, o, lse, ref = attend(M, c, 4, True, max_q)
        check_attention(c, o, lse, ref)
    assert not math.isinf(float(lse[0, 0]))
