"""Accepted paths of more tokens than a list whose places may overlap has elements (128).  Elements beyond that go to other workgroups, and no order
among workgroups is promised, so a longer path moves in calls of up to 128 elements, in ascending order on one stream: element i goes to
base + i and comes from base + m_i with m_i >= i, so no call writes what a later one reads."""
import itertools

import pytest
import torch

import evict_ref as E
from test_evict_gpu import dirty
from test_paged_gpu import Cache

TOGETHER = 128


def path_of(n, m, seed):
    """m of n drafted tokens, ascending."""
    return torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:m].sort().values.to(torch.int32)


def one_call(places, dst, src, order):
    """What a call does to a sequence's places: groups of elements, in some order; each reads all of its own before it writes."""
    for group in order:
        of = slice(group * TOGETHER, (group + 1) * TOGETHER)
        places[dst[of].long()] = places[src[of].long()]


@pytest.mark.parametrize("n, m", [(500, 300), (300, 299), (400, 257)])
def test_calls_of_128_elements_are_needed_and_enough(n, m):
    base, path = 50, path_of(n, m, n)
    before = torch.arange(base + n)
    dst, src = base + torch.arange(m), base + path
    want = before.clone()
    want[dst] = before[src.long()]
    groups = range(-(-m // TOGETHER))
    outcomes = []
    for order in itertools.permutations(groups):
        got = before.clone()
        one_call(got, dst, src, order)
        outcomes.append(torch.equal(got, want))
    assert not all(outcomes)                               # a single call leaves it to the order of the workgroups
    got = before.clone()
    for i in groups:
        of = slice(i * TOGETHER, (i + 1) * TOGETHER)
        one_call(got, dst[of], src[of], [0])
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("D, dt, e4m3", [(64, "bf16", True), (128, "bf16", False), (256, "f16", False)])
def test_a_long_path_moves_in_calls_of_128_elements(D, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    n, m, kvs = 500, 300, [650, 501, 500]
    c = Cache([n] * 3, kvs, 2, D, 16, dt, e4m3, 37)
    dirty(c)
    dst = torch.stack([kv - n + torch.arange(m, dtype=torch.int32) for kv in kvs])[:, None].contiguous()
    src = torch.stack([kv - n + path_of(n, m, b) for b, kv in enumerate(kvs)])[:, None].contiguous()
    dst[1, 0, 290:], src[1, 0, 290:] = -1, -1              # a shorter path
    args, scales = c.on_gpu()
    for i in range(0, m, TOGETHER):
        M.attn_cache_move(*args[:3], dst[..., i:i + TOGETHER].contiguous().cuda(), src[..., i:i + TOGETHER].contiguous().cuda(), **scales)
    as_int = lambda t: t.view(torch.uint8 if c.e4m3 else torch.int16)
    tensors = [as_int(p) for p in c.pages] + [s for s in c.scale if s is not None]
    E.move(tensors, [], c.table, c.page, dst, src)
    for got, want in zip([as_int(p.cpu()) for p in args[:2]] + [s.cpu() for s in scales.values() if s is not None], tensors):
        assert torch.equal(got, want)
