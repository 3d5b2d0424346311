"""Choice among so many places that a workgroup's part of a list is more than it holds at once (lists of more than 64 x 16384 places), against a stable
sort: whole numbers, so equal ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def by_sort(w, kv, keep, stamps, seen, sinks, recent):
    """Dropped places below keep and kept ones from it on, of one list; w has no NaN."""
    number, had = (torch.arange(kv), kv) if stamps is None else (stamps[:kv], seen)
    always = (number < sinks) | (number >= had - recent)
    # tokens that always stay by place, before all others by weight
    order = torch.cat([always.nonzero()[:, 0], torch.where(always, float("-inf"), w[:kv]).sort(descending=True, stable=True).indices])
    order = order[:keep] if int(always.sum()) <= keep else always.nonzero()[:keep, 0]
    kept = torch.zeros(kv, dtype=torch.bool)
    kept[order] = True
    assert int(kept.sum()) == keep
    return (~kept[:keep]).nonzero()[:, 0], kept[keep:].nonzero()[:, 0] + keep


@pytest.mark.parametrize("kind", ["spread", "few", "one"])
@pytest.mark.parametrize("width, kv, keeps", [       # two and three chunks to a part
    (1048592, 1048590, [400001, 1048589, 32768 * 7 + 2]), (2100000, 2099999, [1000003, 5, 49152 * 21 - 3]), (1048592, 1000001, [65536, 999937])])
def test_parts_of_several_chunks(width, kv, keeps, kind):
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(width + kv)
    if kind == "spread":
        w = torch.randn((1, 1, width), generator=gen).mul(2).exp()
    elif kind == "few":
        w = torch.randint(0, 3, (1, 1, width), generator=gen).float()    # ties across chunks and parts
    else:
        w = torch.full((1, 1, width), 0.25)
    stamps = torch.randperm(width + 9, generator=gen)[:width].view(1, 1, width).to(torch.int32)
    i32 = lambda x: torch.tensor([x], dtype=torch.int32)
    dev, dev_stamps = w.cuda(), stamps.cuda()
    for turn, keep in enumerate(keeps):
        for st, seen, sinks, recent in ((None, None, 3, 50), (stamps, width + 9, 1000, 20000)):
            want = by_sort(w[0, 0], kv, keep, None if st is None else st[0, 0], seen, sinks, recent)
            moves = min(keep, kv - keep)
            dst, src, new_len = M.attn_cache_select(dev, i32(kv).cuda(), i32(keep).cuda(), moves, None if st is None else dev_stamps,
                                                    None if st is None else i32(seen).cuda(), sinks=sinks, recent=recent)
            assert new_len.tolist() == [keep]
            for got, x in zip((dst, src), want):
                got = got[0, 0].cpu()
                assert torch.equal(got[:len(x)], x.to(torch.int32)) and (got[len(x):] == -1).all(), (keep, sinks)
