"""Attention over the paged cache where a workgroup's walk is long and where there are more units than workgroups: page windows that
are filled anew several times, missing pages behind the first window, pages beyond 4 GB, second and third passes over the units
with the rings and registers of the first, several row tiles to a sequence.  Against the formula in 64 bits (on the GPU).

What the plan has made of a batch is read from the notes that the kernels leave for the merge in the caller's workspace, so
that a test whose batch is cut in another way fails instead of passing by the mechanism that it is for."""
import math

import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu

GUARD = 4096


class Pool:
    """Pages of a few GB of which a batch uses some, in no order; behind a sequence's last position NaN."""

    def __init__(self, kvs, H, D, page, dt, e4m3, seed, n_pages):
        self.H, self.D, self.page, self.e4m3, self.dt, self.kvs = H, D, page, e4m3, R.DT[dt], kvs
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-kv // page) for kv in kvs]
        self.n_pages = max(n_pages, sum(need) + 1)
        ids = torch.randperm(self.n_pages, generator=gen, device="cuda").int()[:sum(need)]
        ids[0] = self.n_pages - 1 if not (ids == self.n_pages - 1).any() else ids[0]
        self.table = torch.full((len(kvs), max(need) + 1), -1, dtype=torch.int32, device="cuda")
        shape = (self.n_pages, H, page, D)
        self.pages = [torch.empty(shape, dtype=torch.float8_e4m3fn if e4m3 else self.dt, device="cuda") for _ in "kv"]
        self.scale = [torch.empty(shape[:3], dtype=torch.uint8, device="cuda") if e4m3 else None for _ in "kv"]
        at = 0
        for b, n in enumerate(need):
            mine = ids[at:at + n]
            self.table[b, :n] = mine
            at += n
            for i in range(2):
                x = torch.randn((n, H, page, D), generator=gen, device="cuda")
                raw = self.pages[i].view(torch.uint8 if e4m3 else torch.int16)
                x = (x * 128).clamp(-448, 448).to(torch.float8_e4m3fn) if e4m3 else x.to(self.dt)
                bits = x.view(raw.dtype)
                tail = kvs[b] - (n - 1) * page
                if n:
                    bits[-1, :, tail:] = 0x7f if e4m3 else 0x7fff
                raw[mine.long()] = bits
                if e4m3:
                    s = torch.randint(118, 122, (n, H, page), generator=gen, device="cuda", dtype=torch.uint8)
                    if n:
                        s[-1, :, tail:] = 255
                    self.scale[i][mine.long()] = s

    def sequence(self, i, b):
        """Values [H, positions, D] in 64 bits of K (i = 0) or V, and which positions have a page."""
        n = -(-self.kvs[b] // self.page)
        ids = self.table[b, :n]
        ok = (ids >= 0) & (ids < self.n_pages)
        use = ids.clamp(0, self.n_pages - 1).long()
        if self.e4m3:
            x = self.pages[i].view(torch.uint8)[use].view(torch.float8_e4m3fn).double()
            x = x * torch.exp2(self.scale[i][use].double() - 127)[..., None]
        else:
            x = self.pages[i][use].double()
        x = x.transpose(0, 1).reshape(self.H, n * self.page, self.D)[:, :self.kvs[b]]
        return x, ok.repeat_interleave(self.page)[:self.kvs[b]]


def attend(pool, news, G, dt, causal=True):
    """o, lse and the plan's notes (x, y, z, w of every token) of one call with a workspace of exactly its size."""
    from paper_2512_18134_amd import binding as M
    B, T, H_q = len(news), sum(news), pool.H * G
    start = torch.tensor([sum(news[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor(pool.kvs, dtype=torch.int32, device="cuda")
    q = torch.randn((T, H_q, pool.D), generator=pool.gen, device="cuda").to(pool.dt)
    o, lse = torch.full_like(q, float("nan")), torch.full((T, H_q), float("nan"), device="cuda")
    need = M.attn_paged_fwd_workspace_bytes(T, B, H_q, pool.H, pool.D)
    ws = torch.full((need + GUARD,), 0xa5, dtype=torch.uint8, device="cuda")
    entry = M.attn_paged_fwd_f16 if dt == "f16" else M.attn_paged_fwd
    entry(q, *pool.pages, pool.table, start, kv_len, *pool.scale, o=o, lse=lse, workspace=ws[:need], causal=causal, max_q=max(news))
    torch.cuda.synchronize()
    assert (ws[need:] == 0xa5).all(), "written behind the workspace"
    assert B <= 128
    notes = ws[need - 16 * T:need].view(torch.int32).view(T, 4).cpu()
    return q, o, lse, notes


def check(pool, news, G, q, o, lse, dt, causal=True, every=1):
    """Every `every`-th key head against 64 bits, the others for being numbers."""
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    scale, first = 1 / math.sqrt(pool.D), 0
    for b, n in enumerate(news):
        if n == 0:
            continue
        kv = pool.kvs[b]
        (k, ok), (v, _) = pool.sequence(0, b), pool.sequence(1, b)
        j, rows = torch.arange(kv, device="cuda"), torch.arange(n, device="cuda")
        hidden = ~ok[None] | ((j[None] > rows[:, None] + kv - n) if causal else torch.zeros((), dtype=torch.bool, device="cuda"))
        for h in range(0, pool.H, every):
            kt, vh = k[h].T.contiguous(), torch.where(ok[:, None], v[h], 0.0)
            for g in range(G):
                hq = h * G + g
                qh = q[first:first + n, hq].double()
                x = (torch.mm(qh, kt) * scale).masked_fill_(hidden, -math.inf)
                wl = torch.logsumexp(x, -1)
                p = torch.where(hidden, 0.0, torch.exp(x - wl[:, None]))
                wo, weight = torch.mm(p, vh), torch.mm(p, vh.abs())
                size = ((torch.mm(qh.abs(), kt.abs()).masked_fill_(~ok, 0.0).amax(-1)) * scale * (pool.D + 8) + 64) * 2.0 ** -24
                bound = R.bounds(wo, weight, size, R.DT[dt], kv)
                err = (o[first:first + n, hq].double() - wo).abs()
                assert (err <= bound).all(), (b, hq, float((err - bound).max()))
                el = (lse[first:first + n, hq].double() - wl).abs()
                assert (el <= 2 * size + 2e-6 + 2.0 ** -22 * wl.abs()).all(), (b, hq, float(el.max()))
        first += n


def plan_of(notes, news, kvs, H, G, BM):
    """Units of the call and the keys of its longest one, from the notes."""
    units, longest, t = 0, 0, 0
    for n, kv in zip(news, kvs):
        if n:
            _, tiles, ranges, w = notes[t].tolist()
            assert tiles == -(-n * G // BM) and (notes[t:t + n, 1:3] == notes[t, 1:3]).all()
            units += tiles * ranges * H
            longest = max(longest, -(-kv // ranges))
        t += n
    return units, longest


def pages_beyond(H, page, D, e4m3):
    """So many pages that the last one lies more than 2^32 bytes behind the pool's start."""
    return 2 ** 32 // (H * page * D * (1 if e4m3 else 2)) + 37


# ---- tiles: more than 56 (64) of them to a window, three passes and more
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_chunks_whose_windows_are_refilled_and_workgroups_that_take_three_units(D, e4m3, dt):
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    BM = 128 if D == 256 else 256
    n = 2 * BM + 70                                        # three row tiles, the last one ragged
    slots, keys_of_window = (512, 64 * 32) if e4m3 else (256, 56 * (64 if D == 64 else 32))
    long = 2 * keys_of_window + 300
    kvs = [long, long - 77, long - 500, n + 5]
    news = [n, n - 1, n - 60, n]
    H = slots // 4                                         # 12 row tiles to a head: three rounds
    pool = Pool(kvs, H, D, 16, dt, e4m3, 31, pages_beyond(H, 16, D, e4m3))
    # missing: in the first window, next to each other behind it, and at the end of the last one; sequence 1 has all
    pool.table[0, 5] = -1
    pool.table[0, keys_of_window // 16 + 20] = pool.n_pages
    pool.table[2, keys_of_window // 16 + 3] = 2 ** 31 - 1
    pool.table[2, keys_of_window // 16 + 4] = -2 ** 31
    pool.table[2, 2 * keys_of_window // 16 - 1] = -7
    q, o, lse, notes = attend(pool, news, 1, dt)
    units, longest = plan_of(notes, news, kvs, H, 1, BM)
    assert (notes[:, 3] & 1 == 1).all() and units > 2 * slots and longest > 2 * keys_of_window, (units, longest)
    check(pool, news, 1, q, o, lse, dt)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_ranges_of_a_cut_chunk(D, e4m3, causal):
    """One sequence of many keys, cut: walks that begin in the middle of it, with refilled windows, and the merge of their rows."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    BM = 128 if D == 256 else 256
    keys_of_window = 64 * 32 if e4m3 else 56 * (64 if D == 64 else 32)
    kv, n, H, G = 48000 if e4m3 else 28000, BM // 2 * 3, 16, 2               # 3 row tiles of 16 heads
    pool = Pool([kv], H, D, 64, "bf16", e4m3, 32, pages_beyond(H, 64, D, e4m3))
    for i in (11, 60, 61, 200, 333):
        pool.table[0, i] = -1
    q, o, lse, notes = attend(pool, [n], G, "bf16", causal)
    units, longest = plan_of(notes, [n], [kv], H, G, BM)
    assert int(notes[0, 2]) > 1 and longest > keys_of_window, (units, longest)
    check(pool, [n], G, q, o, lse, "bf16", causal)


# ---- rows: 32 steps of a wave to a window, 4096 keys of a workgroup
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
@pytest.mark.parametrize("D, new, G", [(64, 1, 4), (64, 6, 4), (64, 15, 4), (128, 1, 8), (128, 7, 4), (128, 16, 3), (256, 1, 5), (256, 5, 4)],
                         ids=lambda x: str(x))
def test_steps_whose_windows_are_refilled(D, new, G, dt, e4m3):
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    rows = new * G
    BM = 16 if rows <= 16 else 32 if rows <= 32 or D == 256 else 64
    kvs, news = [9000, 8500, 4200, 8200], [new, new, new, max(1, new - 1)]
    H = 136                                                # 544 units: more than run at once
    pool = Pool(kvs, H, D, 32, dt, e4m3, 33, pages_beyond(H, 32, D, e4m3))
    pool.table[0, 40] = -1
    pool.table[0, 4096 // 32 + 9] = pool.n_pages
    pool.table[1, 8192 // 32 + 1] = -2 ** 31
    pool.table[3, 4096 // 32] = -1
    q, o, lse, notes = attend(pool, news, G, dt)
    units, longest = plan_of(notes, news, kvs, H, G, BM)
    assert (notes[:, 3] & 1 == 0).all() and longest > 4096, (units, longest)
    check(pool, news, G, q, o, lse, dt, every=9)


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
@pytest.mark.parametrize("D, new, G", [(D, n, G) for D in (64, 128, 256)
                                       for n, G in ((1, 1), (4, 4), (17, 1), (8, 4), (11, 3), (16, 4), (32, 4))
                                       if n * G <= (64 if D == 256 else 128)], ids=lambda x: str(x))
def test_a_cut_step_keeps_to_its_workspace(D, new, G, dt, e4m3):
    """Partial rows of tiles of 16, 32 and 64 rows, merged; nothing behind the workspace is written, which is as large as the call's
    rows can make it."""
    rows = new * G
    BM = 16 if rows <= 16 else 32 if rows <= 32 or D == 256 else 64
    kvs, news, H = [9001, 2000 + new], [new, max(1, new // 2)], 3
    pool = Pool(kvs, H, D, 16, dt, e4m3, 34, 0)
    q, o, lse, notes = attend(pool, news, G, dt)
    units, longest = plan_of(notes, news, kvs, H, G, BM)
    assert int(notes[0, 2]) > 8, (units, longest)
    check(pool, news, G, q, o, lse, dt)
