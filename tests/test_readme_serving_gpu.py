"""README's calls of a verified tree and of an eviction, run as they stand there, against the plain implementations: the weights that they leave are
those of the accepted tokens, each of which sees what its mask showed it."""
import math
import os
import re
import textwrap

import pytest
import torch

import evict_ref as E
import tree_ref as T
from test_paged_gpu import check_attention

pytestmark = pytest.mark.gpu


def example(entry):
    """The indented lines that import `entry` among others, and what follows them."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        blocks = re.findall(r"(?m)(?:^    .*\n)+", f.read())
    found = [b for b in blocks if re.search(r"import .*\b%s\b" % entry, b)]
    assert len(found) == 1
    return textwrap.dedent(found[0])


def test_a_verified_tree_and_an_eviction():
    B, H, G, D, page, n, m = 3, 2, 4, 128, 16, 20, 6
    gen = torch.Generator().manual_seed(17)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)
    kvs = [320, 45, 700]                                   # with the drafts
    width = 44
    n_pages = B * width
    table = torch.randperm(n_pages, generator=gen).view(B, width).to(torch.int32)
    pages = [torch.randn((n_pages, H, page, D), generator=gen).bfloat16() for _ in "kv"]
    q = torch.randn((B * n, H * G, D), generator=gen).bfloat16()
    start, kv_len = i32([0, n, 2 * n, 3 * n]), i32(kvs)
    # trees whose tokens m_0 < m_1 < ... are a path
    paths = [torch.randperm(n, generator=gen)[:m].sort().values for _ in range(B)]
    sets = []
    for b, path in enumerate(paths):
        of, seen_by = path.tolist(), []
        for i in range(n):
            seen_by.append(sum(1 << j for j in of if j <= i) if i in of else 1 << i)
        sets.append(seen_by)
    mask = T.mask_tensor(B * n, start, sets, 1)
    path = torch.stack(paths).to(torch.int32)
    weights = torch.rand((B, H, width * page), generator=gen)
    stamps = torch.arange(width * page, dtype=torch.int32).expand(B, H, -1).contiguous()
    left = i32([kv - n + m for kv in kvs])
    seen = left + 5
    s = {"torch": torch, "n": n, "m": m, "max_moves": 400}
    for name, t in (("q", q), ("k_pages", pages[0]), ("v_pages", pages[1]), ("page_table", table), ("start", start), ("kv_len", kv_len), ("mask", mask),
                    ("path", path), ("weights", weights), ("stamps", stamps), ("seen", seen), ("keep", i32([300, 31, 400]))):
        s[name] = t.clone().cuda()
    scale = 1 / math.sqrt(D)

    exec(example("attn_paged_tree"), s)
    check = type("Case", (), {"dt": "bf16", "kv_len": kv_len})
    ref = T.attention(q.double(), *(p.double() for p in pages), table, start, kv_len, mask, scale)
    check_attention(check, s["o"].cpu(), s["lse"].cpu(), ref)
    dst = torch.stack([kv - n + torch.arange(m) for kv in kvs])[:, None].to(torch.int32)
    src = torch.stack([kv - n + p for kv, p in zip(kvs, paths)])[:, None].to(torch.int32)
    bits = [p.view(torch.int16) for p in pages]
    E.move(bits, [], table, page, dst, src)
    for got, want in zip((s["k_pages"], s["v_pages"]), bits):
        assert torch.equal(got.cpu().view(torch.int16), want)
    assert torch.equal(s["kv_len"].cpu(), left) and s["kv_len"].dtype == torch.int32
    rows = torch.cat([b * n + p for b, p in enumerate(paths)])
    want, bound, want_stamps = E.weigh(q[rows].double(), s["lse"].cpu()[rows], pages[0].double(), table, i32([0, m, 2 * m, 3 * m]), left, weights,
                                       1.0, True, scale, stamps, seen)
    got = s["weights"].cpu()
    assert ((got.double() - want).abs() <= bound + 1e-30).all() and torch.equal(s["stamps"].cpu(), want_stamps)
    # every accepted row's weights are a distribution over what it sees
    for b in range(B):
        before, k = kvs[b] - n, int(left[b])
        new = got[b, :, :k].double()
        new[:, :before] -= weights[b, :, :before].double()
        assert (new.sum(-1) - m * G).abs().max() < 1e-4 * m * G + k * 2.0 ** -23

    exec(example("attn_cache_select"), s)
    lists = E.select(got, left, i32([300, 31, 400]), 400, want_stamps, seen, sinks=4, recent=256)
    for name, x in zip(("dst", "src", "new_len"), lists):
        assert torch.equal(s[name].cpu(), x)
    beside = [got, want_stamps]
    E.move(bits, beside, table, page, *lists[:2])
    for name, x in (("k_pages", bits[0]), ("v_pages", bits[1]), ("weights", beside[0]), ("stamps", beside[1])):
        have = s[name].cpu()
        assert torch.equal(have.view(torch.int16) if have.dtype == torch.bfloat16 else have, x)
    assert torch.equal(s["kv_len"].cpu(), i32([300, 31, 400]))
