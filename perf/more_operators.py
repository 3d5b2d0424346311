"""What a serving program does with the paged cache besides writing and reading it: attention for trees of drafted tokens, and the
eviction of what attention no longer looks at.

A case is a dict of plain values; its "op" says which call it stands for:
    tree     attn_paged_tree[_f16]: the drafted tokens' queries against their sequence's cache, where a drafted token sees
             its ancestors among the others
    weigh    attn_cache_weigh[_f16]: every cached position's attention weight over the new tokens' queries, added to what it had
    select   attn_cache_select: which places a cache keeps, as moves into the places that become free
    move     attn_cache_move: those moves carried out; or the accepted path of a tree moved to the front of the drafted tokens.
             An e4m3 pool is read back (attn_cache_read[_f16])
Common fields: dtype ("bf16" or "f16": of the rows), B sequences, H_q and H_kv heads, D, page (positions of a page), e4m3 (how the pool
holds its elements), new and kv (the largest sequence's new tokens and cached positions), ragged: "same" (all sequences alike) or
"spread" (kv spread evenly in the logarithm from an eighth of it, new from one token), and
    weigh    decay (of the weights that are there), causal, stamps (token numbers are kept beside the weights)
    select   keep (places of the largest sequence that stay, in proportion of the others), sinks and recent (tokens that stay in any
             case, the first and the last ones), stamps
    move     keep as above and lists for every head; keep = 0: a tree's path of `new` tokens, one list for all heads
"""
import math
import random

import torch

own = False   # False: elementary torch operations; True: this library's entry points

_DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
_DEVICE = "cuda"
_MAX_KV = 131072          # the longest key sequence of this repository's benchmark calls
_MAX_FLOPS = 5.6e11       # a drawn case costs no more than the largest listed ones
_MAX_BYTES = 1.2e9
_MAX_POOL = 1.1e9         # bytes of cache that a case holds
_MAX_SCORES = 1.1e9       # (query, key) pairs that the plain form holds at once


def _case(name, op, dtype, B, new, kv, H_kv, D, page, **more):
    case = {"name": name, "op": op, "dtype": dtype, "e4m3": False, "B": B, "new": new, "kv": kv, "H_q": 0, "H_kv": H_kv, "D": D,
            "page": page, "ragged": "same", "decay": 0.0, "causal": True, "stamps": False, "keep": 0, "sinks": 0, "recent": 0}
    case.update(more)
    return case


def listed():
    return [
        # one sequence, a small tree of drafts: latency is what counts
        _case("tree_one", "tree", "bf16", 1, 15, 1000, 8, 128, 16, H_q=32),
        # a serving batch of ragged lengths, trees of one to 24 drafts, four query heads to a key head
        _case("tree_batch", "tree", "bf16", 32, 24, 8191, 8, 128, 16, H_q=32, ragged="spread"),
        # long contexts in an e4m3 cache, wide trees, eight query heads to a key head: 512 rows on every key
        _case("tree_wide_e4m3", "tree", "bf16", 4, 64, 32768, 8, 128, 64, H_q=64, e4m3=True),
        # wide heads, fp16, an odd number of drafts beyond one word of the mask
        _case("tree_large_heads_f16", "tree", "f16", 16, 77, 2100, 2, 256, 32, H_q=8, ragged="spread"),
        # a decoding step of a full batch adds its weights to what the cache's positions have
        _case("weigh_step", "weigh", "bf16", 64, 1, 8191, 8, 128, 16, H_q=32, ragged="spread", decay=1.0, stamps=True),
        # the last 32 tokens of finished prompts judge the e4m3 cache that the prompts left
        _case("weigh_window_e4m3", "weigh", "f16", 8, 32, 16384, 4, 64, 128, H_q=16, e4m3=True, ragged="spread"),
        # a chunk of a long prompt is weighed whole
        _case("weigh_chunk", "weigh", "bf16", 1, 2048, 16384, 8, 128, 64, H_q=32, decay=0.98),
        # a batch whose caches are 128 places over what they may keep; the newest tokens and the first ones stay
        _case("select_step", "select", "bf16", 64, 1, 2176, 8, 128, 16, keep=2048, sinks=4, recent=256, stamps=True),
        # prompts are cut to a sixteenth
        _case("select_prompts", "select", "bf16", 4, 1, 131072, 8, 128, 256, keep=8192, sinks=4, recent=1024),
        # a verified step: the accepted drafts of 32 trees move up behind the prefix
        _case("move_accepted", "move", "bf16", 32, 5, 4000, 8, 128, 16, ragged="spread"),
        # what select_step has chosen is carried out, weights and token numbers along with it
        _case("move_step_f16", "move", "f16", 64, 1, 2176, 8, 128, 16, keep=2048, stamps=True),
        # prompts in an e4m3 cache are cut to a sixteenth, and what is left is read
        _case("move_prompts_e4m3", "move", "bf16", 4, 1, 131072, 8, 128, 256, keep=8192, e4m3=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["tree", "tree", "weigh", "weigh", "select", "move"])
        D = rng.choice([64, 128, 128, 256])
        H_kv = rng.choice([1, 2, 4, 5, 8, 16])
        H_q = H_kv * rng.choice([1, 2, 3, 4, 8]) if op in ("tree", "weigh") else 0
        B = _log_int(rng, 1, 96)
        kv = _log_int(rng, 1, _MAX_KV)
        case = _case("", op, rng.choice(["bf16", "f16"]), B, 1, kv, H_kv, D, rng.choice([16, 32, 64, 128, 256]), H_q=H_q,
                     ragged=rng.choice(["same", "spread"]))
        if op == "tree":
            case.update(new=min(kv, _log_int(rng, 1, 256)), e4m3=rng.random() < 0.5)
        elif op == "weigh":
            kind = rng.choice(["step", "window", "chunk"])
            new = 1 if kind == "step" else _log_int(rng, 2, 64) if kind == "window" else _log_int(rng, 65, 4096)
            case.update(new=min(kv, new), e4m3=rng.random() < 0.5, decay=rng.choice([0.0, 1.0, 0.95]), causal=rng.random() < 0.8,
                        stamps=rng.random() < 0.5)
        elif op == "select" or rng.random() < 0.6:
            if kv < 16:
                continue
            keep = _log_int(rng, max(1, kv // 32), kv - 1)
            case.update(keep=keep, sinks=min(rng.choice([0, 4, 16]), keep // 4), recent=keep // rng.choice([2, 4, 8, 1000]),
                        stamps=rng.random() < 0.5, e4m3=op == "move" and rng.random() < 0.4)
            if op == "move":
                case.update(sinks=0, recent=0)
        else:
            if kv < 64:
                continue
            case.update(new=rng.randint(1, 8), e4m3=rng.random() < 0.3)
        w = work(case)
        if w["flops"] > _MAX_FLOPS or w["bytes"] > _MAX_BYTES:
            continue
        if op != "select" and _pool_bytes(case) > _MAX_POOL or op in ("tree", "weigh") and _score_count(case) > _MAX_SCORES:
            continue
        if op in ("select", "move") and B * H_kv * kv > 1.8e7:      # (weights that prepare makes and the plain form sorts)
            continue
        del case["name"]
        return case


# ---------------------------------------------------------------------------------------------------------- sizes

_NODES = 64               # drafted tokens of a tree whose accepted path moves


def _lengths(case):
    """(new tokens, cached positions with the new ones) of every sequence: a property of the case, not of the seed."""
    B, new, kv = case["B"], case["new"], case["kv"]
    if case["ragged"] == "same" or B == 1:
        return [new] * B, [kv] * B
    order = list(range(B))
    random.Random(B * 7919 + kv).shuffle(order)
    kvs = [max(1, int(round(kv * 8.0 ** (i / (B - 1) - 1.0)))) for i in order]     # i = B - 1: all of kv
    if case["op"] == "move" and not case["keep"]:
        kvs = [max(k, _NODES) for k in kvs]
    news = [max(1, int(round(new ** (i / (B - 1))))) for i in order]
    return [min(n, k) for n, k in zip(news, kvs)], kvs


def _keeps(case):
    return [k * case["keep"] // case["kv"] for k in _lengths(case)[1]]


def _most_moves(case):
    """Width of the lists of moves: no sequence has more, whatever its weights."""
    if not case["keep"]:
        return case["new"]
    return max(1, max(min(keep, kv - keep) for keep, kv in zip(_keeps(case), _lengths(case)[1])))


def _n_pages(case):
    return sum(-(-k // case["page"]) for k in _lengths(case)[1])


def _width(case):
    return -(-max(_lengths(case)[1]) // case["page"])


def _part_bytes(case):
    """One position of one head in the cache, key or value."""
    return case["D"] + 1 if case["e4m3"] else 2 * case["D"]


def _pool_bytes(case):
    return _n_pages(case) * case["page"] * case["H_kv"] * 2 * _part_bytes(case)


def _pairs(case):
    """(query, key) pairs of one query head; a tree's tokens are taken to see half of the others."""
    n = 0
    for new, kv in zip(*_lengths(case)):
        n += new * kv - (new * (new - 1) // 2 if case["causal"] else 0)
    return n


def _score_count(case):
    news, kvs = _lengths(case)
    return case["B"] * case["H_q"] * max(news) * max(kvs)


def work(case):
    D, H_kv, H_q = case["D"], case["H_kv"], case["H_q"]
    news, kvs = _lengths(case)
    new, kv = sum(news), sum(kvs)
    table = 4 * _n_pages(case)
    q = new * H_q * D * 2
    if case["op"] == "tree":
        words = -(-case["new"] // 64)
        return {"bytes": 2 * q + 4 * new * H_q + 8 * words * new + 2 * kv * H_kv * _part_bytes(case) + table,
                "flops": 4 * D * H_q * _pairs(case)}
    if case["op"] == "weigh":
        old = kv - new if case["decay"] else 0
        return {"bytes": q + 4 * new * H_q + kv * H_kv * _part_bytes(case) + 4 * H_kv * (old + kv + (new if case["stamps"] else 0)) + table,
                "flops": 2 * D * H_q * _pairs(case)}
    if case["op"] == "select":
        lists = 8 * case["B"] * H_kv * _most_moves(case)
        return {"bytes": 4 * H_kv * kv * (2 if case["stamps"] else 1) + lists, "flops": H_kv * kv}
    # (of a head's kept places, as many lie behind the new end as are dropped before it: the expected number of evenly spread ones)
    moved = [keep * (k - keep) // k for keep, k in zip(_keeps(case), kvs)] if case["keep"] else [n - 1 for n in news]
    rows = sum(moved) * H_kv
    heads = H_kv if case["keep"] else 1
    n = 2 * rows * (2 * _part_bytes(case) + (8 if case["stamps"] else 0)) + 8 * heads * case["B"] * _most_moves(case) + table
    if case["e4m3"]:     # the places that stay, read back
        left = sum(_left(case)) * H_kv
        n += 2 * left * (_part_bytes(case) + 2 * D)
    return {"bytes": n, "flops": 0}


def _left(case):
    news, kvs = _lengths(case)
    return _keeps(case) if case["keep"] else [k - _NODES + n if k >= _NODES else k for n, k in zip(news, kvs)]


# ---------------------------------------------------------------------------------------------------------- inputs

def _scale(case):
    return 1.0 / math.sqrt(case["D"])


def _tree_mask(rng, news, words):
    """Random trees: a token's parent is an earlier token of its sequence, or the prefix; a token sees its ancestors and itself."""
    rows = []
    for n in news:
        seen = []
        for i in range(n):
            parent = rng.randint(max(-1, i - 8), i - 1)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        for bits in seen:
            row = [bits >> 64 * w & (1 << 64) - 1 for w in range(words)]
            rows.append([x - (1 << 64) if x >> 63 else x for x in row])
    return torch.tensor(rows, dtype=torch.int64).to(_DEVICE)


def _cache_values(s, n, b):
    """All positions of sequence b, [H_kv, kv, D] in 32 bits."""
    page = s["case"]["page"]
    j = torch.arange(s["kvs"][b], device=_DEVICE)
    ids, at = s["table"][b][j // page].long(), j % page
    return _stored(s[n + "_pages"], s[n + "_scale"], ids, at).transpose(0, 1)


def _input_lse(s, gen):
    """The log-sum-exp that attention has left for the rows."""
    case = s["case"]
    G = case["H_q"] // case["H_kv"]
    lse = torch.empty((s["total"], case["H_q"]), device=_DEVICE)
    for b, (n, kv) in enumerate(zip(s["news"], s["kvs"])):
        k = _cache_values(s, "k", b).transpose(1, 2).contiguous()
        step = max(1, (1 << 28) // (case["H_q"] * kv))
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            rows = slice(s["bounds"][b] + r0, s["bounds"][b] + r1)
            q = s["q"][rows].float().view(r1 - r0, case["H_kv"], G, -1).permute(1, 0, 2, 3).reshape(case["H_kv"], (r1 - r0) * G, -1)
            x = torch.bmm(q, k).mul_(_scale(case)).view(case["H_kv"], r1 - r0, G, kv)
            if case["causal"]:
                last = kv - n + torch.arange(r0, r1, device=_DEVICE)
                x.masked_fill_((torch.arange(kv, device=_DEVICE) > last[:, None])[None, :, None], float("-inf"))
            lse[rows] = torch.logsumexp(x, dim=-1).permute(1, 0, 2).reshape(r1 - r0, -1)
    return lse


def _weights(case, gen):
    """Accumulated weights as attention leaves them: few large ones, many small ones, and some that nothing has looked at."""
    shape = (case["B"], case["H_kv"], _width(case) * case["page"])
    w = torch.randn(shape, generator=gen, device=_DEVICE).mul_(2).exp_().mul_(1e-2)
    return w.mul_(torch.rand(shape, generator=gen, device=_DEVICE) > 0.02)


def _stamps(s, gen):
    """Token numbers of a cache from which half has gone before: the places before the last `recent` hold older tokens in no order.
    Returns the stamps and how many tokens the sequences have had."""
    case = s["case"]
    shape = (case["B"], case["H_kv"], _width(case) * case["page"])
    j = torch.arange(shape[2], device=_DEVICE)
    old = (s["kv_len"] - min(case["recent"] or case["new"], min(s["kvs"]) - 1))[:, None, None]
    r = torch.rand(shape, generator=gen, device=_DEVICE)
    order = torch.where(j < old, r, r + 2).argsort(dim=-1).argsort(dim=-1)
    stamps = torch.where(j < old, 2 * order + (r > 0.5), 2 * old + j - old)
    return stamps.to(torch.int32), (s["kv_len"] + old[:, 0, 0]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed)
    rng = random.Random(seed)
    B, H_q, H_kv, D, page, op = (case[n] for n in ("B", "H_q", "H_kv", "D", "page", "op"))
    dt = _DTYPE[case["dtype"]]
    news, kvs = _lengths(case)
    total, n_pages, width = sum(news), _n_pages(case), _width(case)
    s = {"case": case, "news": news, "kvs": kvs, "total": total, "kv_len": torch.tensor(kvs, dtype=torch.int32, device=_DEVICE)}
    if op == "select":
        s["weights"] = _weights(case, gen)
        s["stamps"], s["seen"] = _stamps(s, gen) if case["stamps"] else (None, None)
        s["keep"] = torch.tensor(_keeps(case), dtype=torch.int32, device=_DEVICE)
        s["moves"] = _most_moves(case)                    # a number of the program's plan, not of a call
        return s

    # a pool in which the sequences' pages lie in no order; the table is padded with -1
    counts = torch.tensor([-(-k // page) for k in kvs], device=_DEVICE)
    ids = torch.randperm(n_pages, generator=gen, device=_DEVICE).to(torch.int32)
    used = torch.arange(width, device=_DEVICE) < counts[:, None]
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device=_DEVICE).masked_scatter_(used, ids)
    s["bounds"] = [sum(news[:b]) for b in range(B + 1)]
    s["start"] = torch.tensor(s["bounds"], dtype=torch.int32, device=_DEVICE)
    for name in "kv" if op != "weigh" else "k":
        pages = torch.empty((n_pages, H_kv, page, D), dtype=torch.float8_e4m3fn if case["e4m3"] else dt, device=_DEVICE)
        step = max(1, (1 << 26) // (H_kv * page * D))
        for i in range(0, n_pages, step):
            x = torch.randn((min(step, n_pages - i), H_kv, page, D), generator=gen, device=_DEVICE)
            # rows of unit variance peak near 3 = 384 * 2^-7
            pages[i:i + step] = x.mul_(128).clamp_(-448, 448).to(pages.dtype) if case["e4m3"] else x.to(dt)
        s[name + "_pages"] = pages
        s[name + "_scale"] = None
        if case["e4m3"]:
            s[name + "_scale"] = torch.randint(119, 122, (n_pages, H_kv, page), generator=gen, device=_DEVICE, dtype=torch.uint8)
    if op in ("tree", "weigh"):
        s["q"] = torch.randn((total, H_q, D), generator=gen, device=_DEVICE).mul_(1.5).to(dt)
    if op == "tree":
        s["mask"] = _tree_mask(rng, news, -(-max(news) // 64))
    elif op == "weigh":
        s["lse"] = _input_lse(s, gen)
        s["weights"] = _weights(case, gen)
        s["out"] = torch.zeros_like(s["weights"])
        s["stamps"], s["seen"] = _stamps(s, gen) if case["stamps"] else (None, None)
    elif case["keep"]:
        s["keep"] = torch.tensor(_keeps(case), dtype=torch.int32, device=_DEVICE)
        weights = _weights(case, gen)
        s["dst"], s["src"], _ = _select_plain({"case": case, "weights": weights, "stamps": None, "kv_len": s["kv_len"], "keep": s["keep"],
                                             "moves": _most_moves(case)})
        s["weights"], s["stamps"] = (weights, _stamps(s, gen)[0]) if case["stamps"] else (None, None)
    else:
        # the accepted path of each tree: its first token is the first drafted one, the others lie behind the path's end
        s["dst"] = torch.full((B, 1, case["new"]), -1, dtype=torch.int32)
        s["src"] = s["dst"].clone()
        for b, (n, kv) in enumerate(zip(news, kvs)):
            if kv >= _NODES:
                path = sorted(rng.sample(range(n, _NODES), n - 1))
                s["dst"][b, 0, :n - 1] = torch.arange(1, n) + kv - _NODES
                s["src"][b, 0, :n - 1] = torch.tensor(path, dtype=torch.int32) + kv - _NODES
        s["dst"], s["src"] = s["dst"].to(_DEVICE), s["src"].to(_DEVICE)
        s["weights"] = s["stamps"] = None
    if op == "move" and case["e4m3"]:
        left = _left(case)
        s["left"] = left
        s["read_start"] = torch.tensor([sum(left[:b]) for b in range(B + 1)], dtype=torch.int32, device=_DEVICE)
        s["read_len"] = torch.tensor(left, dtype=torch.int32, device=_DEVICE)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls

def _entry(name, case):
    from paper_2512_18134_amd import binding
    return getattr(binding, name + ("_f16" if case["dtype"] == "f16" else ""))


def _run_own(s):
    from paper_2512_18134_amd import binding
    case = s["case"]
    if case["op"] == "select":
        dst, src, new_len = binding.attn_cache_select(s["weights"], s["kv_len"], s["keep"], s["moves"], stamps=s["stamps"],
                                                      seen=s["seen"], sinks=case["sinks"], recent=case["recent"])
        return {"dst": dst, "src": src, "new_len": new_len}
    if case["op"] == "tree":
        o, lse = _entry("attn_paged_tree", case)(s["q"], s["k_pages"], s["v_pages"], s["table"], s["start"], s["kv_len"], s["mask"],
                                                 k_scale=s["k_scale"], v_scale=s["v_scale"], scale=_scale(case), max_q=case["new"])
        return {"o": o, "lse": lse}
    if case["op"] == "weigh":
        out = _entry("attn_cache_weigh", case)(s["q"], s["lse"], s["k_pages"], s["table"], s["start"], s["kv_len"], s["weights"],
                                               k_scale=s["k_scale"], out=s["out"], stamps=s["stamps"], seen=s["seen"],
                                               decay=case["decay"], causal=case["causal"], scale=_scale(case), max_q=case["new"])
        return {"weights": out, "stamps": s["stamps"]}
    scales = {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    binding.attn_cache_move(s["k_pages"], s["v_pages"], s["table"], s["dst"], s["src"], **scales, weights=s["weights"],
                            stamps=s["stamps"])
    if not case["e4m3"]:
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights"], "stamps": s["stamps"]}
    k, v = _entry("attn_cache_read", case)(s["k_pages"], s["v_pages"], s["table"], s["read_start"], s["read_len"], sum(s["left"]),
                                           **scales)
    return {"k": k, "v": v}


# ------------------------------------------------------------------------------------------------------ the plain form

def _power(e):
    """2^e in 32 bits, for whole e from -126 to 127."""
    return (e.to(torch.int32) + 127 << 23).view(torch.float32)


def _stored(pages, scale, ids, at):
    """Rows [..., H_kv, D] of the cache in 32 bits, for pages and places [...]."""
    if scale is None:
        return pages[ids, :, at].float()
    x = pages.view(torch.uint8)[ids, :, at].view(torch.float8_e4m3fn)
    return x.float() * _power(scale[ids, :, at].int() - 127)[..., None]


def _all_positions(s):
    """Every sequence's positions up to the longest one: which of them it has, their pages and places."""
    page = s["case"]["page"]
    j = torch.arange(max(s["kvs"]), device=_DEVICE)
    there = j < s["kv_len"][:, None]
    return j, there, s["table"][:, j // page].clamp(min=0).long(), (j % page).expand(len(s["kvs"]), -1)


def _row_index(s):
    """Every sequence's new tokens up to the most of any: which it has, and their rows (row 0 in the place of others)."""
    i = torch.arange(max(s["news"]), device=_DEVICE)
    n = (s["start"][1:] - s["start"][:-1])[:, None]
    there = i < n
    return i, n, there, torch.where(there, s["start"][:-1, None] + i, 0).long()


def _scores(s, k):
    """Scaled scores [B, H_kv, rows, G, positions] in 32 bits."""
    case = s["case"]
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    G = H_q // H_kv
    _, _, _, rows = _row_index(s)
    q = s["q"][rows].float().view(case["B"], -1, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(case["B"] * H_kv, -1, D)
    kt = k.permute(0, 2, 3, 1).reshape(case["B"] * H_kv, D, -1).contiguous()
    return torch.bmm(q, kt).mul_(_scale(case)).view(case["B"], H_kv, -1, G, kt.shape[-1])


def _tree_plain(s):
    case = s["case"]
    B, H_q, H_kv, D = case["B"], case["H_q"], case["H_kv"], case["D"]
    j, there, ids, at = _all_positions(s)
    i, n, mine, _ = _row_index(s)
    x = _scores(s, _stored(s["k_pages"], s["k_scale"], ids, at))
    # the number of a position among the drafted tokens; negative: it lies before them
    node = (j - (s["kv_len"][:, None] - n)).long()[:, None, :].expand(-1, len(i), -1)
    _, _, _, rows = _row_index(s)
    words = s["mask"][rows]
    word = torch.gather(words, 2, (node.clamp(min=0) // 64).clamp(max=words.shape[2] - 1))
    sees = (node < 0) | ((word >> (node.clamp(min=0) % 64)) & 1 == 1) & (node // 64 < words.shape[2])
    sees &= there[:, None, :]
    x.masked_fill_(~sees[:, None, :, None, :], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = _stored(s["v_pages"], s["v_scale"], ids, at).permute(0, 2, 1, 3).reshape(B * H_kv, -1, D).contiguous()
    y = torch.bmm(x.view(B * H_kv, -1, x.shape[-1]), v).view(B, H_kv, len(i), -1, D).div_(total)
    o = y.permute(0, 2, 1, 3, 4).reshape(B, len(i), H_q, D)[mine].to(s["q"].dtype)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, len(i), H_q)[mine]
    return {"o": o, "lse": lse}


def _weigh_plain(s):
    case = s["case"]
    j, there, ids, at = _all_positions(s)
    i, n, mine, rows = _row_index(s)
    x = _scores(s, _stored(s["k_pages"], s["k_scale"], ids, at))
    lse = s["lse"][rows].view(case["B"], len(i), case["H_kv"], -1).permute(0, 2, 1, 3)
    x.sub_(lse[..., None]).exp_()
    first = s["kv_len"][:, None] - n                      # position of the first new token
    last = first + i if case["causal"] else s["kv_len"][:, None].expand(-1, len(i))
    sees = (j <= last[:, :, None]) & mine[:, :, None] & there[:, None, :]
    x.masked_fill_(~sees[:, None, :, None, :], 0.0)
    w = x.sum(dim=(2, 3))
    if case["decay"]:
        w += torch.where((j < first)[:, None], s["weights"][:, :, :len(j)] * case["decay"], 0.0)
    s["out"][:, :, :len(j)] = torch.where(there[:, None], w, s["out"][:, :, :len(j)])
    if case["stamps"]:
        fresh = (j >= first) & there
        number = s["seen"][:, None] - s["kv_len"][:, None] + j
        old = s["stamps"][:, :, :len(j)]
        s["stamps"][:, :, :len(j)] = torch.where(fresh[:, None], number[:, None].to(torch.int32), old)
    return {"weights": s["out"], "stamps": s["stamps"]}


def _select_plain(s):
    """The places of highest weight, ties to the lowest place: a stable sort.  Then the kept places behind the new end go into
    the free ones before it, both in order."""
    case = s["case"]
    w = s["weights"]
    j = torch.arange(w.shape[-1], device=w.device)
    kv, keep = s["kv_len"][:, None, None], s["keep"][:, None, None]
    stamps, seen = (j, kv) if s["stamps"] is None else (s["stamps"], s["seen"][:, None, None])
    always = (stamps < case["sinks"]) | (stamps >= seen - case["recent"])
    w = torch.where(j < kv, torch.where(always, float("inf"), w), -1.0)
    order = w.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, (j < keep).expand_as(w).contiguous())
    M = s["moves"]
    lists = torch.full((2,) + w.shape[:2] + (M + 1,), -1, dtype=torch.int64, device=w.device)
    for i, chosen in enumerate(((j < keep) & ~kept, (j >= keep) & kept)):
        at = torch.where(chosen, chosen.cumsum(dim=-1) - 1, M).clamp(max=M)
        lists[i].scatter_(2, at, j.expand_as(w).contiguous())
    dst, src = lists[..., :M].to(torch.int32).contiguous()
    return dst, src, torch.minimum(s["kv_len"], s["keep"])


def _flat_rows(s, places):
    """Rows of the pool seen as [n_pages * H_kv * page] for places [B, H_kv, M]."""
    case = s["case"]
    b = torch.arange(case["B"], device=_DEVICE)[:, None, None]
    h = torch.arange(case["H_kv"], device=_DEVICE)[:, None]
    p = places.clamp(min=0).long()
    return (s["table"][b, p // case["page"]].long() * case["H_kv"] + h) * case["page"] + p % case["page"]


def _move_plain(s):
    case = s["case"]
    shape = (case["B"], case["H_kv"], s["dst"].shape[2])
    dst, src = s["dst"].expand(shape), s["src"].expand(shape)
    valid = dst >= 0
    to, source = _flat_rows(s, dst)[valid], _flat_rows(s, src)[valid]
    for n in "kv":
        pool = s[n + "_pages"].view(torch.uint8 if case["e4m3"] else _DTYPE[case["dtype"]]).view(-1, case["D"])
        pool[to] = pool[source]
        if case["e4m3"]:
            units = s[n + "_scale"].view(-1)
            units[to] = units[source]
    if case["stamps"]:
        row = torch.arange(shape[0] * shape[1], device=_DEVICE).view(shape[0], shape[1], 1) * s["weights"].shape[-1]
        to, source = (row + dst)[valid].long(), (row + src)[valid].long()
        for x in (s["weights"].view(-1), s["stamps"].view(-1)):
            x[to] = x[source]
    if not case["e4m3"]:
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights"], "stamps": s["stamps"]}
    j = torch.arange(max(s["left"]), device=_DEVICE)
    there = j < s["read_len"][:, None]
    ids, at = s["table"][:, j // case["page"]][there].long(), (j % case["page"]).expand(case["B"], -1)[there]
    return {n: _stored(s[n + "_pages"], s[n + "_scale"], ids, at).to(_DTYPE[case["dtype"]]) for n in "kv"}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "select":
        dst, src, new_len = _select_plain(state)
        return {"dst": dst, "src": src, "new_len": new_len}
    return _tree_plain(state) if op == "tree" else _weigh_plain(state) if op == "weigh" else _move_plain(state)


# ------------------------------------------------------------------------------------------------- the definition, 64 bits

def _exact_rows(s, n, b, count):
    """The first `count` positions of sequence b, [H_kv, count, D] in 64 bits."""
    case = s["case"]
    ids = s["table"][b].long().repeat_interleave(case["page"])[:count]
    at = torch.arange(case["page"], device=_DEVICE).repeat(s["table"].shape[1])[:count]
    if not case["e4m3"]:
        return s[n + "_pages"][ids, :, at].double().permute(1, 0, 2)
    x = s[n + "_pages"].view(torch.uint8)[ids, :, at].view(torch.float8_e4m3fn).double()
    values = torch.tensor([2.0 ** (e - 127) for e in range(256)], dtype=torch.float64, device=_DEVICE)
    return (x * values[s[n + "_scale"][ids, :, at].long()][..., None]).permute(1, 0, 2)


def _exact_tree(case, s):
    G = case["H_q"] // case["H_kv"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device=_DEVICE)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=_DEVICE)
    masks = s["mask"].tolist()
    for b, (n, kv) in enumerate(zip(s["news"], s["kvs"])):
        k, v = _exact_rows(s, "k", b, kv), _exact_rows(s, "v", b, kv)
        rows = slice(s["bounds"][b], s["bounds"][b] + n)
        sees = torch.ones((n, kv), dtype=torch.bool)
        for i, words in enumerate(masks[rows]):
            bits = sum((w % 2 ** 64) << 64 * at for at, w in enumerate(words))
            sees[i, kv - n:] = torch.tensor([bool(bits >> c & 1) for c in range(n)])
        hidden = torch.zeros((n, 1, kv), dtype=torch.float64)
        hidden[:, 0][~sees] = -math.inf
        hidden = hidden.to(_DEVICE)
        for h in range(case["H_kv"]):
            heads = slice(h * G, (h + 1) * G)
            q = s["q"][rows, heads].double().reshape(n * G, -1)
            x = torch.mm(q, k[h].t().contiguous()).view(n, G, kv) * _scale(case) + hidden
            total = torch.logsumexp(x, dim=-1)
            p = torch.exp(x - total[..., None])
            o[rows, heads] = torch.mm(p.view(n * G, kv), v[h].contiguous()).view(n, G, -1)
            lse[rows, heads] = total
    return {"o": o, "lse": lse}


def _exact_weigh(case, s):
    G = case["H_q"] // case["H_kv"]
    w = s["out"].double()
    for b, (n, kv) in enumerate(zip(s["news"], s["kvs"])):
        k = _exact_rows(s, "k", b, kv)
        first = s["bounds"][b]
        for h in range(case["H_kv"]):
            sums = torch.zeros(kv, dtype=torch.float64, device=_DEVICE)
            sums[:kv - n] = s["weights"][b, h, :kv - n].double() * case["decay"]
            step = max(1, (1 << 26) // (kv * G))
            for r in range(0, n, step):
                m = min(step, n - r)
                rows, heads = slice(first + r, first + r + m), slice(h * G, (h + 1) * G)
                x = torch.mm(s["q"][rows, heads].double().reshape(m * G, -1), k[h].t().contiguous()) * _scale(case)
                p = torch.exp(x - s["lse"][rows, heads].double().reshape(m * G, 1)).view(m, G, kv).sum(dim=1)
                if case["causal"]:
                    p = torch.tril(p, diagonal=kv - n + r)
                sums += p.sum(dim=0)
            w[b, h, :kv] = sums
    return {"weights": w, "stamps": None}


def _exact_move(case, s):
    """What lies at every place afterwards, by its index: an untouched place's own, a filled one's source."""
    H, page = case["H_kv"], case["page"]
    source = torch.arange(s["k_pages"].shape[0] * H * page, device=_DEVICE).view(-1, H, page)
    before = source.clone()
    seqs = torch.arange(case["B"], device=_DEVICE)
    for h in range(H):
        of = min(h, s["dst"].shape[1] - 1)
        b, m = torch.nonzero(s["dst"][:, of] >= 0, as_tuple=True)
        d, f = s["dst"][b, of, m].long(), s["src"][b, of, m].long()
        to, come = s["table"][seqs[b], d // page].long(), s["table"][seqs[b], f // page].long()
        source[to, h, d % page] = before[come, h, f % page]
    if case["e4m3"]:
        out = {}
        for n in "kv":
            pages = s[n + "_pages"].view(torch.uint8).view(-1, case["D"])[source].view(s[n + "_pages"].shape)
            moved = {"case": case, "table": s["table"], n + "_pages": pages.view(torch.float8_e4m3fn),
                     n + "_scale": s[n + "_scale"].view(-1)[source]}
            out[n] = torch.cat([_exact_rows(moved, n, b, left).permute(1, 0, 2) for b, left in enumerate(s["left"])])
        return out
    out = {n + "_pages": s[n + "_pages"].view(-1, case["D"])[source].double() for n in "kv"}
    out["weights"] = out["stamps"] = None
    if case["stamps"]:
        w = s["weights"].double()
        for b in range(case["B"]):
            for h in range(H):
                d, f = s["dst"][b, h], s["src"][b, h]
                w[b, h, d[d >= 0].long()] = s["weights"][b, h, f[f >= 0].long()].double()
        out["weights"] = w
    return out


def exact(case, seed):
    if case["op"] == "select":
        return None                                       # whole numbers alone
    s = prepare(case, seed)
    return _exact_tree(case, s) if case["op"] == "tree" else _exact_weigh(case, s) if case["op"] == "weigh" else _exact_move(case, s)
