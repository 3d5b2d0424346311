"""Plain 64-bit implementations of the serving operators (rotary positions, paged cache, attention over it), written
from the formulas of include/attn_rope.h and include/attn_cache.h, on the CPU."""
import math

import torch

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def half_step(dt):
    """A rounding to dt is off by at most this, relative to the value."""
    return torch.finfo(dt).eps / 2


def rope(x, pos, freq, sections, interleaved=False, inverse=False):
    """x [B,H,S,D], pos [axes,B,S], freq [pairs]: float64."""
    pairs = freq.numel()
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)])
    t = pos.double()[axis].permute(1, 2, 0)[:, None] * freq.double()     # [B,1,S,pairs]
    if inverse:
        t = -t
    c, s = t.cos(), t.sin()
    y = x.double().clone()
    i1 = torch.arange(pairs) * 2 if interleaved else torch.arange(pairs)
    i2 = i1 + 1 if interleaved else i1 + pairs
    x1, x2 = x.double()[..., i1], x.double()[..., i2]
    y[..., i1] = x1 * c - x2 * s
    y[..., i2] = x1 * s + x2 * c
    return y


def e4m3_row(x):
    """The values that a row of the cache has in e4m3, and the exponents of its units: x [..., D] -> float64, int."""
    dt = x.dtype
    x = x.double()
    amp = x.abs().amax(-1)
    e = torch.full(amp.shape, -126)
    for k in range(-125, 121):
        e = torch.where(amp > 448 * 2.0 ** (k - 1), torch.full_like(e, k), e)
    unit = torch.tensor(2.0, dtype=torch.float64) ** e[..., None]
    largest = 61440.0 if dt == torch.float16 else 240 * 2.0 ** 120
    y = x.clamp(-largest, largest) / unit
    _, ex = torch.frexp(y)                                   # |y| in [2^(ex-1), 2^ex)
    step = torch.tensor(2.0, dtype=torch.float64) ** (ex - 4).clamp(min=-9)
    return torch.round(y / step) * step * unit, e


def positions(start, kv_len, b):
    n = int(start[b + 1] - start[b])
    return list(range(int(kv_len[b]) - n, int(kv_len[b])))


def place(table, n_pages, page, b, p):
    """(page, place) of a position, or None."""
    if p < 0 or p // page >= table.shape[1]:
        return None
    i = int(table[b, p // page])
    return (i, p % page) if 0 <= i < n_pages else None


def cached(pages, scale):
    x = pages.double() if scale is None else pages.float().double()
    if scale is None:
        return x
    return x * torch.tensor(2.0, dtype=torch.float64) ** (scale.double() - 127)[..., None]


def attention(q, kp, vp, table, start, kv_len, causal, scale):
    """q [T,H_q,D] float64; kp, vp [n_pages,H_kv,page,D]: values of the cache in float64.
    Returns o, lse and, per element of o, sum_j p_j |v_j| and a bound on the error of a score; rows of nobody: NaN."""
    T, H_q, D = q.shape
    n_pages, H_kv, page, _ = kp.shape
    G = H_q // H_kv
    nan = float("nan")
    o, weight = torch.full((T, H_q, D), nan, dtype=torch.float64), torch.zeros((T, H_q, D), dtype=torch.float64)
    lse, size = torch.full((T, H_q), nan, dtype=torch.float64), torch.zeros((T, H_q), dtype=torch.float64)
    for b in range(len(kv_len)):
        first, n, kv = int(start[b]), int(start[b + 1] - start[b]), min(int(kv_len[b]), table.shape[1] * page)
        at = [place(table, n_pages, page, b, p) for p in range(kv)]
        keys = torch.tensor([p for p in range(kv) if at[p] is not None], dtype=torch.long)
        if n == 0:
            continue
        if len(keys) == 0:
            o[first:first + n], lse[first:first + n] = 0, -math.inf
            continue
        ids, pl = (torch.tensor([at[p][i] for p in keys.tolist()]) for i in (0, 1))
        k, v = kp[ids, :, pl], vp[ids, :, pl]                 # [keys,H_kv,D]
        for h in range(H_q):
            kh, vh, qh = k[:, h // G], v[:, h // G], q[first:first + n, h]
            x = qh @ kh.T * scale
            rows = torch.arange(n)[:, None] + kv - n
            if causal:
                x = x.masked_fill(keys[None] > rows, -math.inf)
            top = x.amax(-1, keepdim=True)
            ok = torch.isfinite(top)
            p = torch.where(ok, (x - torch.where(ok, top, 0.0)).exp(), torch.zeros_like(x))
            total = p.sum(-1, keepdim=True)
            p = torch.where(ok, p / total.clamp(min=1e-300), torch.zeros_like(p))
            o[first:first + n, h] = p @ vh
            weight[first:first + n, h] = p @ vh.abs()
            lse[first:first + n, h] = torch.where(ok, top + total.clamp(min=1e-300).log(), torch.full_like(top, -math.inf))[:, 0]
            # fp32 accumulation of D products, a few roundings of the scaled score
            size[first:first + n, h] = ((qh.abs() @ kh.abs().T).amax(-1) * scale * (D + 8) + 64) * 2.0 ** -24
    return o, lse, weight, size


def bounds(o, weight, size, dt, n_keys):
    """How far o may be off: each P is off by half a step and by its score's error, o by half a step of its own (P below the
    smallest normal number of fp16: by 2^-25)."""
    h = half_step(dt)
    tiny = n_keys * 2.0 ** -25 if dt == torch.float16 else 0.0
    return h * o.abs() * (1 + h) + weight * (h + 2 * size[..., None] + 1e-6) + tiny * weight.amax()
