"""A plain 64-bit implementation of the attention of drafted tokens over the paged cache, from the formula of include/attn_tree.h, on
the CPU; masks as sets of bits."""
import math
import random

import torch

import serving_ref as R


def words(bits, n):
    """`bits`, a Python integer, as n words of 64 bits in int64."""
    row = [bits >> 64 * w & (1 << 64) - 1 for w in range(n)]
    return [x - (1 << 64) if x >> 63 else x for x in row]


def random_tree(n, seed):
    """Ancestor sets, as integers, of n tokens: a token's parent is an earlier one of the last nine, or the prefix."""
    rng, seen = random.Random(seed), []
    for i in range(n):
        parent = rng.randint(max(-1, i - 9), i - 1)
        seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
    return seen


def lower_triangle(n):
    return [(2 << i) - 1 for i in range(n)]


def mask_tensor(T, start, sets, n_words, fill=-1):
    """[T, n_words] int64: sets[b][i] is what row start[b] + i sees; rows of nobody are `fill`."""
    rows = [[fill] * n_words for _ in range(T)]
    for b, of in enumerate(sets):
        for i, bits in enumerate(of):
            rows[int(start[b]) + i] = words(bits, n_words)
    return torch.tensor(rows, dtype=torch.int64).reshape(T, n_words)


def attention(q, kp, vp, table, start, kv_len, mask, scale):
    """As serving_ref.attention, with mask [T, words]."""
    T, H_q, D = q.shape
    n_pages, H_kv, page, _ = kp.shape
    G = H_q // H_kv
    nan = float("nan")
    o, weight = torch.full((T, H_q, D), nan, dtype=torch.float64), torch.zeros((T, H_q, D), dtype=torch.float64)
    lse, size = torch.full((T, H_q), nan, dtype=torch.float64), torch.zeros((T, H_q), dtype=torch.float64)
    for b in range(len(kv_len)):
        first, n, kv = int(start[b]), int(start[b + 1] - start[b]), min(int(kv_len[b]), table.shape[1] * page)
        if n == 0:
            continue
        at = [R.place(table, n_pages, page, b, p) for p in range(kv)]
        keys = [p for p in range(kv) if at[p] is not None]
        if not keys:
            o[first:first + n], lse[first:first + n] = 0, -math.inf
            continue
        ids, pl = (torch.tensor([at[p][i] for p in keys]) for i in (0, 1))
        k, v = kp[ids, :, pl], vp[ids, :, pl]                 # [keys,H_kv,D]
        hidden = torch.zeros((n, len(keys)), dtype=torch.bool)
        for i in range(n):
            bits = sum((w % 2 ** 64) << 64 * x for x, w in enumerate(mask[first + i].tolist()))
            hidden[i] = torch.tensor([p >= kv - n and not bits >> (p - (kv - n)) & 1 for p in keys])
        for h in range(H_q):
            kh, vh, qh = k[:, h // G], v[:, h // G], q[first:first + n, h]
            x = (qh @ kh.T * scale).masked_fill(hidden, -math.inf)
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
