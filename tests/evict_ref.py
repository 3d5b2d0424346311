"""Plain implementations of attn_cache_weigh, attn_cache_select and attn_cache_move, from the formulas of include/attn_evict.h, on the
CPU, place by place."""
import math

import torch

import serving_ref as R


def weigh(q, lse, kp, table, start, kv_len, weights, decay, causal, scale, stamps=None, seen=None):
    """float64 weights [B,H_kv,L] (places that are not written: as in `weights`), and per place a bound on the relative error of its
    sum: a score is off by fp32 accumulation of D products and a few roundings of numbers as large as itself and lse."""
    T, H_q, D = q.shape
    n_pages, H_kv, page, _ = kp.shape
    G = H_q // H_kv
    L = table.shape[1] * page
    out, bound = weights.double().clone(), torch.zeros(weights.shape, dtype=torch.float64)
    new_stamps = None if stamps is None else stamps.clone()
    for b in range(len(kv_len)):
        first, n, kv = int(start[b]), int(start[b + 1] - start[b]), min(max(int(kv_len[b]), 0), L)
        if n <= 0 or kv == 0:
            continue
        at = [R.place(table, n_pages, page, b, p) for p in range(kv)]
        there = torch.tensor([a is not None for a in at])
        ids, pl = (torch.tensor([a[i] if a else 0 for a in at]) for i in (0, 1))
        j = torch.arange(kv)
        own = j >= kv - n
        for h in range(H_kv):
            k = torch.where(there[:, None], kp[ids, h, pl], 0.0)
            w, err = torch.zeros(kv, dtype=torch.float64), torch.zeros(kv, dtype=torch.float64)
            for g in range(G):
                qh, ls = q[first:first + n, h * G + g], lse[first:first + n, h * G + g].double()
                sees = (ls != -math.inf)[:, None] & there[None]
                if causal:
                    sees &= j[None] <= kv - n + torch.arange(n)[:, None]
                x = qh @ k.T * scale
                ls = torch.where(ls == -math.inf, 0.0, ls)
                p = torch.where(sees, (x - ls[:, None]).exp(), 0.0)
                size = (qh.abs() @ k.abs().T * scale * (D + 8) + ls.abs()[:, None] * 4 + 8) * 2.0 ** -24
                w += p.sum(0)
                err += (p * size).sum(0)
            # fp32 sums of n G terms, all positive; exp2's own error
            err += w * ((n * G + 8) * 2.0 ** -24 + 2.0 ** -22)
            old = torch.zeros(kv, dtype=torch.float64) if decay == 0 else torch.where(own, 0.0, weights[b, h, :kv].double() * decay)
            out[b, h, :kv] = old + w
            bound[b, h, :kv] = err + (old + w) * 2.0 ** -22
            if stamps is not None:
                new_stamps[b, h, :kv][own] = (int(seen[b]) - kv + j[own]).to(torch.int32)
    return out, bound, new_stamps


def select(weights, kv_len, keep, moves, stamps=None, seen=None, sinks=0, recent=0):
    B, H, width = weights.shape
    dst, src = torch.full((B, H, moves), -1, dtype=torch.int32), torch.full((B, H, moves), -1, dtype=torch.int32)
    new_len = torch.empty(B, dtype=torch.int32)
    for b in range(B):
        kv = min(max(int(kv_len[b]), 0), width)
        end = min(kv, max(int(keep[b]), 0))
        if min(end, kv - end) > moves:
            new_len[b] = kv
            continue
        new_len[b] = end
        for h in range(H):
            w = weights[b, h, :kv].tolist()
            number = list(range(kv)) if stamps is None else stamps[b, h, :kv].tolist()
            had = kv if seen is None else int(seen[b])
            always = [n < sinks or n >= had - recent for n in number]
            order = sorted(range(kv), key=lambda j: (not always[j], (-math.inf if always[j] else w[j] != w[j]),
                                                      0.0 if always[j] or w[j] != w[j] else -w[j], j))
            kept = set(order[:end])
            holes = [j for j in range(end) if j not in kept]
            movers = [j for j in range(end, kv) if j in kept]
            assert len(holes) == len(movers)
            dst[b, h, :len(holes)] = torch.tensor(holes, dtype=torch.int32)
            src[b, h, :len(movers)] = torch.tensor(movers, dtype=torch.int32)
    return dst, src, new_len


def move(tensors, rows, table, page, dst, src):
    """tensors: [n_pages, H, page, ...] of the cache; rows: [B, H, L] beside it.  Sources are read before anything is written."""
    before = [t.clone() for t in tensors], [t.clone() for t in rows]
    n_pages, H = tensors[0].shape[:2]
    for b in range(dst.shape[0]):
        for h in range(H):
            of = 0 if dst.shape[1] == 1 else h
            for d, s in zip(dst[b, of].tolist(), src[b, of].tolist()):
                to, come = R.place(table, n_pages, page, b, d), R.place(table, n_pages, page, b, s)
                if to is None or come is None:
                    continue
                for t, old in zip(tensors, before[0]):
                    t[to[0], h, to[1]] = old[come[0], h, come[1]]
                for t, old in zip(rows, before[1]):
                    t[b, h, d] = old[b, h, s]
