"""Rotary positions in calls with so many tokens that a wave takes several heads with its sines, and with outputs that are stored past
the caches: heads that are no multiple of what a wave takes or has in flight, waves that go from q to k, parts of a head, strides, in
place.  Against the formula in 64 bits (on the GPU).  test_serving_launches.py holds these sizes to the kernels that they are for."""
import pytest
import torch

import serving_ref as R
from test_rope_gpu import entry

pytestmark = pytest.mark.gpu

SIZES = [  # B, H_q, H_kv, S, D, sections, heads of a wave, stored past the caches
    (1, 6, 3, 32771, 64, [32], 8, False),                  # 9 heads: a wave's second group has one, q ends inside the first
    (3, 5, 2, 10923, 64, [8, 16, 0, 8], 4, False),
    (2, 3, 3, 21000, 64, [5, 3], 1, False),                # 8 of 32 pairs: a lane to a token
    (1, 13, 4, 16389, 128, [20, 28], 16, True),            # 17 heads: 48 of 64 pairs
    (2, 30, 3, 8191, 128, [16, 24, 24], 16, True),
    (1, 21, 0, 33000, 64, [32], 16, True),                 # q alone
    (1, 7, 7, 10001, 256, [32, 8], 4, True),               # 40 of 128 pairs, 5 lanes of 8
]


def tensors(size, dt, seed=7):
    b, hq, hkv, s, d, sections, _, _ = size
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (torch.randn(b, h, s, d, generator=gen, device="cuda").to(R.DT[dt]) for h in (hq, hkv))
    pos = torch.randint(-5, 131072, (len(sections), b, s), generator=gen, device="cuda", dtype=torch.int32)
    n = sum(sections)
    return q, k if hkv else None, pos, 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)


def check(got, x, pos, freq, sections, inter, inverse, dt):
    """The bound of test_rope_gpu.check, eight heads at a time."""
    for h in range(0, x.shape[1], 8):
        part = x[:, h:h + 8]
        want = R.rope(part, pos, freq, sections, inter, inverse)
        bound = R.half_step(R.DT[dt]) * want.abs() + 1e-6 * part.double().abs().amax(-1, keepdim=True) * 2
        err = (got[:, h:h + 8].double() - want).abs()
        assert (err <= bound).all(), (h, float((err - bound).max()))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "B%d_H%d_%d_S%d_D%d" % s[:5])
def test_large_calls_match_the_formula(size, inter, inverse):
    from paper_2512_18134_amd import binding as M
    dt = "f16" if inter == inverse else "bf16"
    q, k, pos, freq = tensors(size, dt)
    sections = size[5]
    yq, yk = entry(M, dt)(q, k, pos, freq, sections, interleaved=inter, inverse=inverse)
    check(yq, q, pos, freq, sections, inter, inverse, dt)
    if k is None:
        assert yk is None
        return
    check(yk, k, pos, freq, sections, inter, inverse, dt)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("size", [SIZES[0], SIZES[3]], ids=lambda s: "D%d" % s[4])
def test_large_calls_in_place_and_on_slices_of_rows(size, inter):
    """The same bits as the plain call: q and k as slices of a projection's rows, turned in place and into a second tensor's slices."""
    from paper_2512_18134_amd import binding as M
    q, k, pos, freq = tensors(size, "bf16")
    b, hq, hkv, s, d, sections, _, _ = size
    want = M.attn_rope(q, k, pos, freq, sections, interleaved=inter)
    view = lambda t, first, n: t[:, first:first + n].transpose(0, 1)[None]
    rows = torch.zeros(s, hq + hkv + 2, d, dtype=torch.bfloat16, device="cuda")
    rows[:, -2:] = 3.0
    view(rows, 0, hq).copy_(q), view(rows, hq, hkv).copy_(k)
    other = torch.full_like(rows, 5.0)
    M.attn_rope(view(rows, 0, hq), view(rows, hq, hkv), pos, freq, sections, q_out=view(other, 0, hq), k_out=view(other, hq, hkv),
                interleaved=inter)
    assert torch.equal(view(other, 0, hq), want[0]) and torch.equal(view(other, hq, hkv), want[1]) and (other[:, -2:] == 5).all()
    assert torch.equal(view(rows, 0, hq), q) and torch.equal(view(rows, hq, hkv), k)
    M.attn_rope(view(rows, 0, hq), view(rows, hq, hkv), pos, freq, sections, q_out=view(rows, 0, hq), k_out=view(rows, hq, hkv),
                interleaved=inter)
    assert torch.equal(view(rows, 0, hq), want[0]) and torch.equal(view(rows, hq, hkv), want[1]) and (rows[:, -2:] == 3).all()
