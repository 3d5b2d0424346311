"""Serving a language model next to this library's attention: rotary positions of several axes, a paged cache of keys and
values (written in 16 bits or in e4m3, and read back) and the attention of new tokens over that cache.

A case is a dict of plain values; its "op" says which call it stands for:
    rope     attn_rope[_f16]: q and k turned by their positions; with grad the gradients of both are turned back as well
    write    attn_cache_write[_f16]: the new tokens' keys and values into their pages; the whole pool is the output.  A pool
             in e4m3 is read back (attn_cache_read[_f16]) at the places that were written
    read     attn_cache_read[_f16]: the last positions of every sequence back into rows
    attend   attn_paged_fwd[_f16]: the new tokens' queries against all keys of their sequence
Common fields: dtype ("bf16" or "f16"), D, H_kv, and
    rope     B, S, H_q, axes, rot (rotated elements of a head), interleaved, fused (slices of one projection's rows), grad
    others   B sequences; e4m3 (how the pool holds its elements), page (positions of a page), new and kv: the sizes of the
             largest sequence's new tokens and of its cache; ragged: "same" (all sequences alike), "spread" (kv spread evenly
             in the logarithm from an eighth of it, new from one token), "one" (one sequence has all of new, the others one token)
"""
import math
import random

import torch

own = False   # False: elementary torch operations; True: this library's entry points

_DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
_DEVICE = "cuda"
_MAX_KV = 131072          # the longest key sequence of this repository's benchmark calls
_MAX_FLOPS = 1.2e12       # a drawn case costs no more than the largest listed ones
_MAX_BYTES = 1.5e9
_MAX_POOL = 1.1e9         # bytes of cache that a case reads


def _rope(name, dtype, B, S, H_q, H_kv, D, axes, rot, interleaved=False, fused=False, grad=False):
    return {"name": name, "op": "rope", "dtype": dtype, "B": B, "S": S, "H_q": H_q, "H_kv": H_kv, "D": D, "axes": axes,
            "rot": rot, "interleaved": interleaved, "fused": fused, "grad": grad}


def _cache(name, op, dtype, e4m3, B, new, kv, H_kv, D, page, ragged, H_q=0, causal=True):
    return {"name": name, "op": op, "dtype": dtype, "e4m3": e4m3, "B": B, "new": new, "kv": kv, "H_q": H_q, "H_kv": H_kv,
            "D": D, "page": page, "ragged": ragged, "causal": causal}


def listed():
    return [
        # one decoding step of 64 sequences: q and k are slices of the projection's rows; three axes (time, height, width)
        _rope("rope_step", "bf16", 1, 64, 32, 8, 128, 3, 128, fused=True),
        # an attention layer of a training step on image patches: forward and the way back
        _rope("rope_train", "bf16", 4, 4096, 16, 16, 128, 3, 128, grad=True),
        # a text model that turns half of every head, in neighbouring pairs, on a prompt of an odd length
        _rope("rope_prompt_f16", "f16", 2, 777, 16, 4, 64, 1, 32, interleaved=True),
        # a decoding step leaves 64 new rows in the cache
        _cache("write_step", "write", "bf16", False, 64, 1, 512, 8, 128, 16, "spread"),
        # prompts enter an e4m3 cache; the rows as it holds them come back, for a prefix that the dense forward takes
        _cache("write_prompts_e4m3", "write", "f16", True, 4, 4096, 4096, 8, 128, 64, "spread"),
        # a short 16-bit prefix, and long e4m3 ones, back in rows
        _cache("read_prefix", "read", "f16", False, 2, 300, 300, 4, 64, 16, "same"),
        _cache("read_long_e4m3", "read", "bf16", True, 8, 16384, 16384, 8, 128, 128, "spread"),
        # one sequence decodes: latency is what counts
        _cache("attend_one", "attend", "bf16", False, 1, 1, 1000, 16, 64, 16, "same", H_q=16),
        # a full serving batch of ragged lengths, four query heads to a key head
        _cache("attend_batch", "attend", "bf16", False, 64, 1, 8191, 8, 128, 16, "spread", H_q=32),
        # few sequences of the longest context, e4m3 cache
        _cache("attend_long_e4m3", "attend", "bf16", True, 4, 1, 131072, 8, 128, 256, "same", H_q=64),
        # four drafted tokens of every sequence are scored at once, wide heads
        _cache("attend_drafts_f16", "attend", "f16", False, 16, 4, 4100, 2, 256, 32, "spread", H_q=8),
        # a chunk of a long prompt against everything before it
        _cache("attend_chunk", "attend", "bf16", False, 1, 2048, 32768, 8, 128, 64, "same", H_q=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    H_kv = rng.choice([1, 2, 4, 5, 8, 16])
    return H_kv, H_kv * rng.choice([1, 2, 3, 4, 8])


def draw(rng):
    while True:
        op = rng.choice(["rope", "write", "read", "attend", "attend"])
        D = rng.choice([64, 128, 128, 256])
        dtype = rng.choice(["bf16", "f16"])
        H_kv, H_q = _heads(rng)
        if op == "rope":
            axes = rng.choice([1, 2, 3])
            case = _rope("", dtype, rng.choice([1, 1, 2, 3, 4]), _log_int(rng, 1, 16384), H_q, H_kv, D, axes,
                         rng.choice([D, D, D // 2]), rng.random() < 0.3, rng.random() < 0.5, rng.random() < 0.5)
            case["fused"] = case["fused"] and case["B"] == 1
        else:
            B = _log_int(rng, 1, 96)
            kv = _log_int(rng, 1, _MAX_KV)
            kind = rng.choice(["step", "drafts", "chunk"])
            new = 1 if kind == "step" else _log_int(rng, 2, 8) if kind == "drafts" else _log_int(rng, 16, 4096)
            ragged = rng.choice(["same", "spread", "one"])
            if op == "read":
                new = kv
                ragged = rng.choice(["same", "spread"])
            case = _cache("", op, dtype, rng.random() < 0.5, B, min(new, kv), kv, H_kv, D, rng.choice([16, 32, 64, 128, 256]),
                          ragged, H_q if op == "attend" else 0, op != "attend" or rng.random() < 0.85)
        w = work(case)
        if w["flops"] > _MAX_FLOPS or w["bytes"] > _MAX_BYTES or ("kv" in case and _pool_bytes(case) > _MAX_POOL):
            continue
        if case["op"] == "attend" and _score_count(case) > 4e9:
            continue
        del case["name"]
        return case


# ---------------------------------------------------------------------------------------------------------- sizes

def _lengths(case):
    """(new tokens, cached positions with the new ones) of every sequence: a property of the case, not of the seed."""
    B, new, kv = case["B"], case["new"], case["kv"]
    if case["ragged"] == "same" or B == 1:
        return [new] * B, [kv] * B
    order = list(range(B))
    random.Random(B * 7919 + kv).shuffle(order)
    kvs = [max(1, int(round(kv * 8.0 ** (i / (B - 1) - 1.0)))) for i in order]     # i = B - 1: all of kv
    if case["ragged"] == "one":
        news = [new if i == B - 1 else 1 for i in order]
    elif case["op"] == "read":
        news = list(kvs)
    else:
        news = [max(1, int(round(new ** (i / (B - 1))))) for i in order]
        if case["op"] == "write" and new == kv:
            news = list(kvs)
    return [min(n, k) for n, k in zip(news, kvs)], kvs


def _n_pages(case):
    return sum(-(-k // case["page"]) for k in _lengths(case)[1])


def _row_bytes(case):
    """One position of one head in the cache, key and value."""
    return 2 * (case["D"] + 1) if case["e4m3"] else 4 * case["D"]


def _pool_bytes(case):
    return _n_pages(case) * case["page"] * case["H_kv"] * _row_bytes(case)


def _pairs(case):
    """(query, key) pairs that the mask leaves, for one query head."""
    n = 0
    for new, kv in zip(*_lengths(case)):
        n += new * kv - (new * (new - 1) // 2 if case["causal"] else 0)
    return n


def _score_count(case):
    return case["H_q"] * sum(n * k for n, k in zip(*_lengths(case)))


def work(case):
    D, H_kv = case["D"], case["H_kv"]
    if case["op"] == "rope":
        heads = case["H_q"] + case["H_kv"]
        rows = case["B"] * case["S"]
        passes = 2 if case["grad"] else 1
        once = rows * (heads * 2 * 2 * D + 4 * case["axes"])
        return {"bytes": passes * once, "flops": passes * rows * heads * 3 * case["rot"]}
    new, kv = (sum(x) for x in _lengths(case))
    rows16 = new * H_kv * 4 * D
    table = 4 * _n_pages(case)
    if case["op"] == "write":
        stored = new * H_kv * _row_bytes(case)
        # read back: the stored rows once more, and the rows
        return {"bytes": rows16 + stored + (stored + rows16 if case["e4m3"] else 0) + 4 * new,
                "flops": 2 * new * H_kv * 2 * D if case["e4m3"] else 0}
    if case["op"] == "read":
        return {"bytes": rows16 + new * H_kv * _row_bytes(case) + table, "flops": 2 * new * H_kv * D if case["e4m3"] else 0}
    q = new * case["H_q"] * D * 2
    return {"bytes": 2 * q + 4 * new * case["H_q"] + kv * H_kv * _row_bytes(case) + table,
            "flops": 4 * D * case["H_q"] * _pairs(case)}


# ---------------------------------------------------------------------------------------------------------- inputs

def _scale(case):
    return 1.0 / math.sqrt(case["D"])


def _sections(case):
    """How many pairs of a head follow each axis: the first axis (time) has the fewest."""
    pairs, axes = case["rot"] // 2, case["axes"]
    rest = [pairs * 3 // 8] * (axes - 1) if axes == 3 else [pairs // 2] * (axes - 1)
    return [pairs - sum(rest)] + rest


def _prepare_rope(case, gen):
    B, S, H_q, H_kv, D, axes = (case[n] for n in ("B", "S", "H_q", "H_kv", "D", "axes"))
    dt = _DTYPE[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=_DEVICE, dtype=torch.float32).to(dt)
    state = {}
    if case["fused"]:
        rows = normal(S, H_q + 2 * H_kv, D)
        state["q"] = rows[:, :H_q].transpose(0, 1)[None]
        state["k"] = rows[:, H_q:H_q + H_kv].transpose(0, 1)[None]
    else:
        state["q"], state["k"] = normal(B, H_q, S, D), normal(B, H_kv, S, D)
    if case["grad"]:
        state["dq"], state["dk"] = normal(B, H_q, S, D), normal(B, H_kv, S, D)
    if axes == 1:
        # a prompt that continues at some place of a long context
        first = torch.randint(0, _MAX_KV, (B, 1), generator=gen, device=_DEVICE)
        pos = (first + torch.arange(S, device=_DEVICE))[None]
    elif case["grad"]:
        # patches of a picture: one time, rows, columns
        side = max(1, math.isqrt(S))
        i = torch.arange(S, device=_DEVICE) + torch.randint(0, 64, (B, 1), generator=gen, device=_DEVICE)
        pos = torch.stack([torch.zeros_like(i), i // side, i % side][3 - axes:])
    else:
        # tokens of different sequences, each with its own place on every axis
        pos = torch.randint(0, _MAX_KV, (axes, B, S), generator=gen, device=_DEVICE)
    state["pos"] = pos.to(torch.int32).contiguous()
    half = case["rot"] // 2
    state["freq"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=_DEVICE) / half)
    state["sections"] = _sections(case)
    return state


def _prepare_cache(case, gen):
    B, H_q, H_kv, D, page = (case[n] for n in ("B", "H_q", "H_kv", "D", "page"))
    dt = _DTYPE[case["dtype"]]
    news, kvs = _lengths(case)
    total, n_pages = sum(news), _n_pages(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=_DEVICE, dtype=torch.float32).to(dt)

    # a pool in which the sequences' pages lie in no order; the table is padded with -1
    width = max(-(-k // page) for k in kvs)
    ids = torch.randperm(n_pages, generator=gen, device=_DEVICE).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=_DEVICE)
    at = 0
    for b, kv in enumerate(kvs):
        n = -(-kv // page)
        table[b, :n] = ids[at:at + n]
        at += n
    state = {"news": news, "kvs": kvs, "table": table, "total": total}
    bounds = [0]
    for n in news:
        bounds.append(bounds[-1] + n)
    state["start"] = torch.tensor(bounds, dtype=torch.int32, device=_DEVICE)
    state["bounds"] = bounds
    state["kv_len"] = torch.tensor(kvs, dtype=torch.int32, device=_DEVICE)
    for name in ("k", "v"):
        pages = torch.empty((n_pages, H_kv, page, D), dtype=torch.float8_e4m3fn if case["e4m3"] else dt, device=_DEVICE)
        step = max(1, (1 << 26) // (H_kv * page * D))
        for i in range(0, n_pages, step):
            x = torch.randn((min(step, n_pages - i), H_kv, page, D), generator=gen, device=_DEVICE)
            # rows of unit variance peak near 3 = 384 * 2^-7
            pages[i:i + step] = x.mul_(128).clamp_(-448, 448).to(pages.dtype) if case["e4m3"] else x.to(dt)
        state[name + "_pages"] = pages
        state[name + "_scale"] = None
        if case["e4m3"]:
            state[name + "_scale"] = torch.randint(119, 122, (n_pages, H_kv, page), generator=gen, device=_DEVICE,
                                                   dtype=torch.uint8)
    if case["op"] == "write":
        # rows of different sizes, as activations are
        size = torch.exp(torch.randn((total, H_kv, 1), generator=gen, device=_DEVICE)).to(dt)
        state["k"], state["v"] = normal(total, H_kv, D) * size, normal(total, H_kv, D) * size
    elif case["op"] == "attend":
        state["q"] = normal(total, H_q, D)
    return state


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed)
    state = _prepare_rope(case, gen) if case["op"] == "rope" else _prepare_cache(case, gen)
    state["case"] = case
    return state


# ------------------------------------------------------------------------------------------------ the library's calls

def _entry(name, case):
    from paper_2512_18134_amd import binding
    return getattr(binding, name + ("_f16" if case["dtype"] == "f16" else ""))


def _run_own(s):
    case = s["case"]
    if case["op"] == "rope":
        rope = _entry("attn_rope", case)
        q, k = rope(s["q"], s["k"], s["pos"], s["freq"], s["sections"], interleaved=case["interleaved"])
        out = {"q": q, "k": k}
        if case["grad"]:
            out["dq"], out["dk"] = rope(s["dq"], s["dk"], s["pos"], s["freq"], s["sections"], interleaved=case["interleaved"],
                                        inverse=True)
        return out
    cache = (s["k_pages"], s["v_pages"], s["table"], s["start"], s["kv_len"])
    scales = {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if case["op"] == "attend":
        o, lse = _entry("attn_paged_fwd", case)(s["q"], *cache, **scales, causal=case["causal"], scale=_scale(case),
                                                max_q=case["new"])
        return {"o": o, "lse": lse}
    if case["op"] == "write":
        _entry("attn_cache_write", case)(s["k"], s["v"], *cache, **scales)
        if not case["e4m3"]:
            return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    k, v = _entry("attn_cache_read", case)(*cache, s["total"], **scales)
    return {"k": k, "v": v}


# ------------------------------------------------------------------------------------------------------ the plain form

def _angles(pos, freq, sections):
    """cos and sin [B, S, pairs] in 32 bits, of angles in 64."""
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    angle = pos[axis].double().permute(1, 2, 0) * freq
    return angle.cos().float(), angle.sin().float()


def _turn(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    y = x.float().clone()
    c, s = cos[:, None], sin[:, None]
    if interleaved:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    else:
        a, b = slice(0, rot // 2), slice(rot // 2, rot)
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a] = xa * c - xb * s
    y[..., b] = xa * s + xb * c
    return y.to(x.dtype)


def _places(s, b):
    """(page, place in the page) of the positions of sequence b's new rows."""
    page = s["case"]["page"]
    p = torch.arange(s["kvs"][b] - s["news"][b], s["kvs"][b], device=_DEVICE)
    return s["table"][b][p // page].long(), p % page


def _power(e):
    """2^e in 32 bits, for whole e from -126 to 127."""
    return (e.to(torch.int32) + 127 << 23).view(torch.float32)


def _quantise(x):
    """Rows as e4m3 and the power of two that they are multiples of: the smallest that brings the largest element to 448 or
    less, an exponent of 8 bits.  x is multiplied exactly; what would read back as infinity stays one step below."""
    top = 61440.0 if x.dtype == torch.float16 else 240.0 * 2.0 ** 120
    x = x.float()
    mant, expo = torch.frexp(x.abs().amax(dim=-1))              # mant in [0.5, 1), or 0
    e = (expo - 9 + (mant > 0.875).to(expo.dtype)).clamp(-126, 120)
    e = torch.where(mant == 0, torch.full_like(e, -126), e)
    q = (x.clamp(-top, top) * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8)


def _stored(pages, scale, ids, at):
    """Rows [n, H_kv, D] of the cache in 32 bits."""
    if scale is None:
        return pages[ids, :, at].float()
    x = pages.view(torch.uint8)[ids, :, at].view(torch.float8_e4m3fn)
    return x.float() * _power(scale[ids, :, at].int() - 127)[..., None]


def _write_plain(s):
    for b in range(len(s["news"])):
        ids, at = _places(s, b)
        rows = slice(s["bounds"][b], s["bounds"][b + 1])
        for n in ("k", "v"):
            x = s[n][rows]
            if s[n + "_scale"] is not None:
                x, s[n + "_scale"][ids, :, at] = _quantise(x)
            if x.dtype == torch.float8_e4m3fn:
                s[n + "_pages"].view(torch.uint8)[ids, :, at] = x.view(torch.uint8)
            else:
                s[n + "_pages"][ids, :, at] = x


def _read_plain(s):
    case = s["case"]
    out = {n: torch.empty((s["total"], case["H_kv"], case["D"]), dtype=_DTYPE[case["dtype"]], device=_DEVICE) for n in "kv"}
    for b in range(len(s["news"])):
        ids, at = _places(s, b)
        for n in "kv":
            out[n][s["bounds"][b]:s["bounds"][b + 1]] = _stored(s[n + "_pages"], s[n + "_scale"], ids, at).to(out[n].dtype)
    return out


def _attend_plain(s):
    case = s["case"]
    H_q, H_kv, D, page = case["H_q"], case["H_kv"], case["D"], case["page"]
    G = H_q // H_kv
    o = torch.empty_like(s["q"])
    lse = torch.empty((s["total"], H_q), device=_DEVICE)
    for b, (n, kv) in enumerate(zip(s["news"], s["kvs"])):
        j = torch.arange(kv, device=_DEVICE)
        ids, at = s["table"][b][j // page].long(), j % page
        kt = _stored(s["k_pages"], s["k_scale"], ids, at).permute(1, 2, 0).contiguous()       # [H_kv, D, kv]
        v = _stored(s["v_pages"], s["v_scale"], ids, at).transpose(0, 1).contiguous()         # [H_kv, kv, D]
        step = max(1, (1 << 28) // (H_q * kv))
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            rows = slice(s["bounds"][b] + r0, s["bounds"][b] + r1)
            q = s["q"][rows].float().view(r1 - r0, H_kv, G, D).permute(1, 0, 2, 3).reshape(H_kv, (r1 - r0) * G, D)
            x = torch.bmm(q, kt).mul_(_scale(case))
            if case["causal"] and r0 + 1 < n:
                last = kv - n + torch.arange(r0, r1, device=_DEVICE).repeat_interleave(G)
                x.masked_fill_(j > last[:, None], float("-inf"))
            top = x.amax(dim=-1, keepdim=True)
            x.sub_(top).exp_()
            total = x.sum(dim=-1, keepdim=True)
            y = torch.bmm(x, v).div_(total)
            o[rows] = y.view(H_kv, r1 - r0, G, D).permute(1, 0, 2, 3).reshape(r1 - r0, H_q, D).to(o.dtype)
            lse[rows] = (top + total.log()).view(H_kv, r1 - r0, G).permute(1, 0, 2).reshape(r1 - r0, H_q)
    return {"o": o, "lse": lse}


def _run_plain(s):
    case = s["case"]
    if case["op"] == "rope":
        cos, sin = _angles(s["pos"], s["freq"], s["sections"])
        out = {n: _turn(s[n], cos, sin, case["interleaved"]) for n in ("q", "k")}
        if case["grad"]:     # the turn is orthogonal: its gradient is the turn back
            cos, sin = _angles(s["pos"], s["freq"], s["sections"])
            out.update({n: _turn(s[n], cos, -sin, case["interleaved"]) for n in ("dq", "dk")})
        return out
    if case["op"] == "attend":
        return _attend_plain(s)
    if case["op"] == "write":
        _write_plain(s)
        if not case["e4m3"]:
            return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return _read_plain(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------- the definition, 64 bits

def _as_complex(x, interleaved, rot):
    x = x.double()[..., :rot]
    if interleaved:
        return torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous())
    return torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:].contiguous())


def _exact_rope(case, s):
    """A pair is a complex number and the turn a multiplication by exp(i angle)."""
    rot, out = case["rot"], {}
    angle = torch.empty((case["B"], 1, case["S"], rot // 2), dtype=torch.float64, device=_DEVICE)
    first = 0
    for a, n in enumerate(s["sections"]):
        angle[:, 0, :, first:first + n] = s["pos"][a].double()[:, :, None] * s["freq"][first:first + n]
        first += n
    unit = torch.polar(torch.ones_like(angle), angle)
    for name in ("q", "k") + (("dq", "dk") if case["grad"] else ()):
        z = _as_complex(s[name], case["interleaved"], rot) * (unit.conj() if name[0] == "d" else unit)
        parts = torch.view_as_real(z)
        turned = parts.flatten(-2) if case["interleaved"] else torch.cat([parts[..., 0], parts[..., 1]], dim=-1)
        out[name] = torch.cat([turned, s[name].double()[..., rot:]], dim=-1)
    return out


def _exact_e4m3(x):
    """The value that a row's elements have in the cache: multiples of the row's power of two, rounded to three bits behind
    the leading one (ties to even), and to multiples of 2^-9 below 2^-6."""
    top = 61440.0 if x.dtype == torch.float16 else 240.0 * 2.0 ** 120
    x = x.double()
    size = x.abs().amax(dim=-1, keepdim=True)
    unit = torch.full_like(size, 2.0 ** -126)
    for e in (128, 64, 32, 16, 8, 4, 2, 1):                     # the smallest power of two that 448 times reaches size
        larger = unit * 2.0 ** (e - 1)
        unit = torch.where(size > larger * 448, larger * 2, unit)
    y = x.clamp(-top, top) / unit
    step = torch.full_like(y, 2.0 ** -9)
    for e in range(-5, 9):
        step = torch.where(y.abs() >= 2.0 ** e, 2.0 ** (e - 3), step)
    return torch.round(y / step) * step * unit


def _flat_places(case, s):
    """For every new row: its page and its place in the page, all sequences at once."""
    news, kvs = torch.tensor(s["news"]), torch.tensor(s["kvs"])
    seq = torch.repeat_interleave(torch.arange(case["B"]), news)
    row = torch.arange(s["total"]) - torch.tensor(s["bounds"][:-1])[seq]
    pos = (kvs[seq] - news[seq] + row).to(_DEVICE)
    return s["table"][seq.to(_DEVICE), pos // case["page"]].long(), pos % case["page"]


def _exact_rows(case, s, n, ids, at):
    if not case["e4m3"]:
        return s[n + "_pages"][ids, :, at].double()
    x = s[n + "_pages"].view(torch.uint8)[ids, :, at].view(torch.float8_e4m3fn).double()
    values = torch.tensor([2.0 ** (e - 127) for e in range(256)], dtype=torch.float64, device=_DEVICE)
    return x * values[s[n + "_scale"][ids, :, at].long()][..., None]


def _exact_attend(case, s):
    H_q, H_kv, page = case["H_q"], case["H_kv"], case["page"]
    if _score_count(case) > 4e9:
        return None
    G = H_q // H_kv
    o = torch.empty(s["q"].shape, dtype=torch.float64, device=_DEVICE)
    lse = torch.empty((s["total"], H_q), dtype=torch.float64, device=_DEVICE)
    for b, (n, kv) in enumerate(zip(s["news"], s["kvs"])):
        pos = torch.arange(kv, device=_DEVICE)
        ids = s["table"][b].long().repeat_interleave(page)[:kv]
        k, v = (_exact_rows(case, s, x, ids, pos % page) for x in "kv")
        first = s["bounds"][b]
        for h in range(H_kv):
            kh, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
            step = max(1, (1 << 27) // (kv * G))
            for r in range(0, n, step):
                m = min(step, n - r)
                q = s["q"][first + r:first + r + m, h * G:(h + 1) * G].double().reshape(m * G, -1)
                x = torch.mm(q, kh) * _scale(case)
                if case["causal"]:
                    seen = kv - n + r + torch.arange(m, device=_DEVICE)
                    x = torch.where(pos[None, None] <= seen[:, None, None], x.view(m, G, kv), -math.inf).view(m * G, kv)
                total = torch.logsumexp(x, dim=-1)
                o[first + r:first + r + m, h * G:(h + 1) * G] = torch.mm(torch.exp(x - total[:, None]), vh).view(m, G, -1)
                lse[first + r:first + r + m, h * G:(h + 1) * G] = total.view(m, G)
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] == "attend":
        return _exact_attend(case, s)
    ids, at = _flat_places(case, s)
    if case["op"] == "read":
        return {n: _exact_rows(case, s, n, ids, at) for n in "kv"}
    if case["e4m3"]:
        return {n: _exact_e4m3(s[n]) for n in "kv"}
    out = {}
    for n in "kv":
        pages = s[n + "_pages"].double()
        pages[ids, :, at] = s[n].double()
        out[n + "_pages"] = pages
    return out
