"""attn_rope[_f16] against the formula in 64 bits: axes, partial turns, both pairings, strides, far positions, in place; and its
backward against the formula's gradient and differences."""
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def entry(B, dt):
    return B.attn_rope_f16 if dt == "f16" else B.attn_rope


def inputs(B, H_q, H_kv, S, D, sections, dt, seed, far=131072):
    gen = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(B, h, S, D, generator=gen).to(R.DT[dt]) for h in (H_q, H_kv))
    pos = torch.randint(-5, far, (len(sections), B, S), generator=gen, dtype=torch.int32)
    n = sum(sections)
    return q, k, pos, 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)


def check(got, want, x, dt, name):
    """One rounding of the result; the 32-bit sine, cosine (angle to 2^-25 turns), products and sum: below 1e-6 of the pair."""
    bound = R.half_step(R.DT[dt]) * want.abs() + 1e-6 * x.double().abs().amax(-1, keepdim=True) * 2
    err = (got.cpu().double() - want).abs()
    assert (err <= bound).all(), (name, float((err - bound).max()))


CASES = [  # B, H_q, H_kv, S, D, sections, interleaved
    (1, 1, 1, 1, 64, [32], False),
    (1, 32, 8, 64, 128, [16, 24, 24], False),
    (2, 3, 1, 77, 128, [64], True),
    (3, 5, 5, 130, 64, [8, 0, 8], False),          # half of a head, an axis without pairs
    (1, 4, 2, 33, 256, [32, 96], True),
    (2, 2, 1, 9, 256, [8], False),                 # one chunk of a head
    (1, 7, 7, 513, 128, [5, 7, 11, 1], False),     # sections that end inside a lane's pairs; 48 of 128 elements
    (1, 2, 2, 4099, 128, [40], True),              # 5 lanes of 8
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_rope_matches_the_formula(case, dt):
    from paper_2512_18134_amd import binding as M
    b, hq, hkv, s, d, sections, inter = case
    q, k, pos, freq = inputs(b, hq, hkv, s, d, sections, dt, 3)
    dev = [t.cuda() for t in (q, k, pos, freq)]
    for inverse in (False, True):
        yq, yk = entry(M, dt)(*dev, sections, interleaved=inter, inverse=inverse)
        check(yq, R.rope(q, pos, freq, sections, inter, inverse), q, dt, "q")
        check(yk, R.rope(k, pos, freq, sections, inter, inverse), k, dt, "k")
    only, none = entry(M, dt)(dev[0], None, *dev[2:], sections, interleaved=inter)
    again, _ = entry(M, dt)(*dev, sections, interleaved=inter)
    assert none is None and torch.equal(only, again)


def test_positions_far_beyond_any_context_keep_their_angle():
    """2^31 - 1 times a frequency of 1: 64-bit products leave 2^-22 of a turn, 1.5e-6 radians."""
    from paper_2512_18134_amd import binding as M
    q, k, pos, freq = inputs(1, 2, 1, 64, 64, [32], "f16", 4)
    pos = (2 ** 31 - 1 - torch.arange(64, dtype=torch.int64) * 30000001).to(torch.int32)[None, None]
    yq, _ = M.attn_rope_f16(q.cuda(), k.cuda(), pos.cuda(), freq.cuda(), [32])
    want = R.rope(q, pos, freq, [32])
    bound = R.half_step(torch.float16) * want.abs() + 5e-6 * q.double().abs().amax(-1, keepdim=True)
    assert ((yq.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("layout", ["fused rows", "rows out", "in place", "broadcast input", "token slices"])
def test_strides(layout):
    from paper_2512_18134_amd import binding as M
    hq, hkv, s, d, sections = 6, 2, 37, 128, [8, 24]
    gen = torch.Generator().manual_seed(5)
    rows = torch.randn(s, hq + 2 * hkv, d, generator=gen).bfloat16()
    pos = torch.randint(0, 9999, (2, 1, s), generator=gen, dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    on = rows.cuda()
    view = lambda t, a, b: t[:, a:b].transpose(0, 1)[None]
    q, k = view(on, 0, hq), view(on, hq, hq + hkv)
    wq, wk = (R.rope(view(rows, a, b), pos, freq, sections) for a, b in ((0, hq), (hq, hq + hkv)))
    args = (pos.cuda(), freq.cuda(), sections)
    xq, xk = view(rows, 0, hq), view(rows, hq, hq + hkv)
    if layout == "fused rows":
        yq, yk = M.attn_rope(q, k, *args)
    elif layout == "rows out":
        out = torch.full((s, hq + hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        yq, yk = M.attn_rope(q, k, *args, q_out=view(out, 0, hq), k_out=view(out, hq, hq + hkv))
        assert torch.isfinite(out.float()).all()
    elif layout == "in place":
        yq, yk = M.attn_rope(q, k, *args, q_out=q, k_out=k)
        assert torch.equal(on[:, hq + hkv:].cpu(), rows[:, hq + hkv:])        # the values between them are not touched
    elif layout == "broadcast input":
        q1 = q[:, :1].expand(1, hq, s, d)
        yq, yk = M.attn_rope(q1, k, *args)
        xq = xq[:, :1].expand(1, hq, s, d)
        wq = R.rope(xq, pos, freq, sections)
    else:
        yq, yk = M.attn_rope(q[:, :, ::2], k[:, :, ::2], args[0][:, :, ::2].contiguous(), *args[1:])
        wq, wk, xq, xk = wq[:, :, ::2], wk[:, :, ::2], xq[:, :, ::2], xk[:, :, ::2]
    check(yq, wq, xq, "bf16", "q")
    check(yk, wk, xk, "bf16", "k")


@pytest.mark.parametrize("inter", [False, True])
def test_the_turn_back_is_the_gradient(inter):
    """Against the formula's gradient by automatic differentiation in 64 bits, and against differences: for a linear map
    <g, y(x + h)> - <g, y(x)> = <dx, h> whatever the size of h."""
    from paper_2512_18134_amd import binding as M
    sections = [16, 8, 8]
    q, k, pos, freq = inputs(2, 4, 2, 45, 64, sections, "f16", 6)
    g = [torch.randn(t.shape, generator=torch.Generator().manual_seed(7)).half() for t in (q, k)]
    leaves = [t.double().requires_grad_() for t in (q, k)]
    sum((R.rope(x, pos, freq, sections, inter) * y.double()).sum() for x, y in zip(leaves, g)).backward()
    dev = (pos.cuda(), freq.cuda(), sections)
    dx = M.attn_rope_f16(g[0].cuda(), g[1].cuda(), *dev, interleaved=inter, inverse=True)
    for got, x, y in zip(dx, leaves, g):
        check(got, x.grad, y, "f16", "dx")
    h = [torch.randn(t.shape, generator=torch.Generator().manual_seed(8)).half() for t in (q, k)]
    y0 = M.attn_rope_f16(q.cuda(), k.cuda(), *dev, interleaved=inter)
    moved = [(x.double() + d.double()).half() for x, d in zip((q, k), h)]
    y1 = M.attn_rope_f16(moved[0].cuda(), moved[1].cuda(), *dev, interleaved=inter)
    for i in range(2):
        step = moved[i].double() - (q, k)[i].double()
        change = (g[i].double() * (y1[i].cpu().double() - y0[i].cpu().double())).sum()
        slope = (dx[i].cpu().double() * step).sum()
        # each of three tensors is rounded by half a step of its own element
        rounding = R.half_step(torch.float16) * ((g[i].double() * y1[i].cpu().double()).abs().sum() +
                                                 (g[i].double() * y0[i].cpu().double()).abs().sum() +
                                                 (dx[i].cpu().double() * step).abs().sum())
        assert (change - slope).abs() <= rounding * 1.01


def test_refusals():
    from paper_2512_18134_amd import binding as M
    q, k, pos, freq = (t.cuda() for t in inputs(1, 2, 1, 5, 64, [32], "bf16", 1))
    with pytest.raises(TypeError):
        M.attn_rope_f16(q, k, pos, freq, [32])
    with pytest.raises(TypeError):
        M.attn_rope(q, k, pos.long(), freq, [32])
    with pytest.raises(TypeError):
        M.attn_rope(q, k, pos, freq.float(), [32])
    with pytest.raises(TypeError):
        M.attn_rope(q, k, pos, freq, [16, 16])
    with pytest.raises(ValueError):
        M.attn_rope(q, k[:, :, :4], pos, freq, [32])
    with pytest.raises(TypeError):
        M.attn_rope(q.transpose(2, 3), k, pos, freq, [32])
    with pytest.raises(ValueError):
        M.attn_rope(q, k, pos, freq, [32], q_out=q[:, :1].expand(1, 2, 5, 64))
    with pytest.raises(M.AttnError):
        M.attn_rope(q, k, pos, freq[:12].contiguous(), [12])
