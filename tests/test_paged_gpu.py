"""The paged cache and the attention over it against plain implementations in 64 bits: types, kinds, head layouts, page sizes,
lengths from nothing to several ranges, ragged batches, padding, strides, bad pages."""
import math

import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def fn(M, name, dt):
    return getattr(M, name + ("_f16" if dt == "f16" else ""))


class Cache:
    """A pool filled with noise (places of nobody with NaN), a shuffled page table padded with -1, lengths."""

    def __init__(self, news, kvs, H_kv, D, page, dt, e4m3, seed, front=0, behind=0, spare=3):
        gen = torch.Generator().manual_seed(seed)
        self.gen, self.dt, self.e4m3, self.page, self.H_kv, self.D = gen, dt, e4m3, page, H_kv, D
        need = [-(-kv // page) for kv in kvs]
        self.n_pages = max(1, sum(need) + spare)
        ids = torch.randperm(self.n_pages, generator=gen).to(torch.int32)
        self.table = torch.full((len(kvs), max(1, max(need)) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.start = torch.tensor([front + sum(news[:b]) for b in range(len(news) + 1)], dtype=torch.int32)
        self.kv_len = torch.tensor(kvs, dtype=torch.int32)
        self.T = front + sum(news) + behind
        shape = (self.n_pages, H_kv, page, D)
        self.scale = [None, None]
        if e4m3:
            self.pages = [(torch.randn(shape, generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in "kv"]
            self.scale = [torch.randint(117, 123, shape[:3], generator=gen, dtype=torch.uint8) for _ in "kv"]
        else:
            self.pages = [torch.randn(shape, generator=gen).to(R.DT[dt]) for _ in "kv"]
        used = torch.zeros(shape[:3], dtype=torch.bool)
        for b, kv in enumerate(kvs):
            for i in range(need[b]):
                used[self.table[b, i].long(), :, :min(page, kv - i * page)] = True
        for i in range(2):
            if e4m3:
                self.pages[i].view(torch.uint8)[~used] = 0x7f          # NaN
                self.scale[i][~used] = 255
            else:
                self.pages[i][~used] = float("nan")

    def values(self):
        return [R.cached(p, s) for p, s in zip(self.pages, self.scale)]

    def on_gpu(self):
        if not hasattr(self, "_gpu"):
            self._gpu = [t.cuda() for t in self.pages], [None if s is None else s.cuda() for s in self.scale]
            self._index = [t.cuda() for t in (self.table, self.start, self.kv_len)]
        return self._gpu[0] + self._index, dict(k_scale=self._gpu[1][0], v_scale=self._gpu[1][1])

    def rows(self, H):
        return torch.randn((self.T, H, self.D), generator=self.gen).to(R.DT[self.dt])


def attend(M, c, G, causal=True, max_q=None, q=None):
    q = c.rows(c.H_kv * G) if q is None else q
    scale = 1 / math.sqrt(c.D)
    args, scales = c.on_gpu()
    o = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    ws = torch.full((M.attn_paged_fwd_workspace_bytes(c.T, len(c.kv_len), q.shape[1], c.H_kv, c.D) // 4,), float("nan"),
                    device="cuda")
    got = fn(M, "attn_paged_fwd", c.dt)(q.cuda(), *args, **scales, o=o, lse=lse, workspace=ws, causal=causal, max_q=max_q)
    assert got[0] is o and got[1] is lse
    torch.cuda.synchronize()
    return q, o.cpu(), lse.cpu(), R.attention(q.double(), *c.values(), c.table, c.start, c.kv_len, causal, scale)


def check_attention(c, o, lse, ref):
    wo, wl, weight, size = ref
    mine = ~torch.isnan(wl)
    assert torch.isnan(lse[~mine]).all() and torch.isnan(o[~mine].float()).all(), "rows of nobody were written"
    bound = R.bounds(wo, weight, size, R.DT[c.dt], max(1, int(c.kv_len.max())))
    err = (o.double() - wo).abs()
    assert (err[mine] <= bound[mine]).all(), float((err - bound)[mine].max())
    empty = mine & torch.isinf(wl)
    assert (lse[empty] == -math.inf).all() and (o[empty] == 0).all()
    full = mine & ~empty
    el = (lse.double() - wl).abs()[full]
    assert (el <= 2 * size[full] + 2e-6 + 2.0 ** -22 * wl[full].abs()).all(), float(el.max())


SHAPES = [  # news, kvs, H_kv, G, D, page
    ([1], [1], 1, 1, 64, 16),
    ([1], [1000], 3, 1, 64, 16),
    ([1] * 5, [17, 1, 300, 64, 129], 2, 4, 128, 16),
    ([1, 1], [2300, 70], 1, 8, 128, 256),
    ([1], [700], 2, 5, 256, 32),
    ([1], [33], 1, 40, 128, 64),                          # 40 query heads on one key head
    ([4] * 3, [400, 4, 131], 2, 3, 128, 32),              # drafted tokens
    ([3, 0, 1, 7], [90, 50, 1, 1030], 2, 4, 256, 16),
    ([5, 1], [5, 6], 2, 16, 64, 128),
    ([100], [100], 2, 4, 128, 16),                        # a prompt from its start
    ([130, 1, 37], [500, 777, 37], 1, 2, 64, 64),
    ([65], [1200], 2, 1, 256, 128),
    ([300], [2500], 1, 4, 128, 32),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n%s_kv%s_H%d_G%d_D%d_p%d" % (max(s[0]), max(s[1]), *s[2:]))
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
def test_attention_matches_the_formula(shape, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    news, kvs, H, G, D, page = shape
    c = Cache(news, kvs, H, D, page, dt, e4m3, 11, front=2, behind=3)
    q = None
    for causal in (True, False):
        q, o, lse, ref = attend(M, c, G, causal, max(news), q)
        check_attention(c, o, lse, ref)


@pytest.mark.parametrize("max_q", [1, 3, 9, 1000, None])
def test_the_hint_costs_speed_only(max_q):
    from paper_2512_18134_amd import binding as M
    c = Cache([1, 40, 9, 0, 2], [300, 40, 2000, 16, 77], 2, 128, 16, "bf16", False, 12)
    _, o, lse, ref = attend(M, c, 4, True, max_q)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", True)])
@pytest.mark.parametrize("most", [3, 50])
def test_batches_of_many_sequences(most, dt, e4m3):
    """So many that the cut is worked out before the kernels that take its units; of few rows, or of few and of many."""
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(17)
    news = torch.randint(0, 4, (150,), generator=gen).tolist()
    kvs = [n + int(torch.randint(0, 60, (1,), generator=gen)) for n in news]
    news[70], kvs[70], kvs[71], kvs[149] = most, 700, 1500, 300
    c = Cache(news, kvs, 2, 64, 16, dt, e4m3, 18, front=1, behind=2)
    for max_q in (most, None):
        _, o, lse, ref = attend(M, c, 3, True, max_q)
        check_attention(c, o, lse, ref)


@pytest.mark.parametrize("long", [700, 8000])
def test_more_sequences_than_the_cut_takes_at_once(long):
    """More than the 1024 lanes that work the cut out, one of them cut into ranges."""
    from paper_2512_18134_amd import binding as M
    gen = torch.Generator().manual_seed(19)
    news = torch.randint(0, 2, (2100,), generator=gen).tolist()
    kvs = [n + int(torch.randint(0, 30, (1,), generator=gen)) for n in news]
    news[1500], kvs[1500] = 1, long
    c = Cache(news, kvs, 1, 64, 16, "bf16", False, 20)
    _, o, lse, ref = attend(M, c, 2, True, 1)
    check_attention(c, o, lse, ref)


@pytest.mark.parametrize("n", [1, 70])
def test_rows_that_see_nothing(n):
    from paper_2512_18134_amd import binding as M
    c = Cache([n, n, n], [0, max(1, n - 30), 500], 2, 64, 16, "f16", False, 13)
    for causal in (True, False):
        _, o, lse, ref = attend(M, c, 2, causal, n)
        check_attention(c, o, lse, ref)
    assert torch.isinf(ref[1][:n]).all()


@pytest.mark.parametrize("n, e4m3", [(1, False), (1, True), (80, False), (80, True)])
def test_bad_pages_are_not_seen(n, e4m3):
    """Page numbers outside the pool, lengths beyond the table: their keys are invisible, and nothing else is touched."""
    from paper_2512_18134_amd import binding as M
    c = Cache([n, n, n], [900, 333, 100], 2, 128, 16, "bf16", e4m3, 14)
    c.table[0, 3] = -1
    c.table[0, 10:14] = c.n_pages
    c.table[0, 20] = 2 ** 31 - 1
    c.table[1, :] = -2 ** 31                  # no page at all
    c.kv_len[2] = 2 ** 31 - 1                 # ends where the table does; every place up to there that has a page is seen
    for i, x in enumerate(c.pages):
        if e4m3:
            x.view(torch.uint8)[x.view(torch.uint8) & 0x7f == 0x7f] = 0x38
            c.scale[i][c.scale[i] == 255] = 120
        else:
            x[torch.isnan(x)] = 1.0
    _, o, lse, _ = attend(M, c, 4, True, n, q := c.rows(8))
    known = c.kv_len.clone()
    known[2] = c.table.shape[1] * 16
    ref = R.attention(q.double(), *c.values(), c.table, c.start, known, True, 1 / math.sqrt(128))
    check_attention(c, o, lse, ref)
    assert torch.isinf(lse[n:2 * n]).all()


def test_queries_and_keys_in_slices_of_projected_rows():
    from paper_2512_18134_amd import binding as M
    c = Cache([4, 1, 20], [100, 64, 20], 2, 128, 16, "bf16", False, 15)
    rows = torch.randn(c.T, 8 + 2 + 2, 128, generator=c.gen).bfloat16()
    dev = rows.cuda()
    args, _ = c.on_gpu()
    M.attn_cache_write(dev[:, 8:10], dev[:, 10:12], *args)
    for i in range(2):
        c.pages[i] = c._gpu[0][i].cpu()
    for b in range(3):
        for i, p in enumerate(R.positions(c.start, c.kv_len, b)):
            page, at = R.place(c.table, c.n_pages, 16, b, p)
            t = int(c.start[b]) + i
            assert torch.equal(c.pages[0][page, :, at], rows[t, 8:10]) and torch.equal(c.pages[1][page, :, at], rows[t, 10:12])
    o, lse = M.attn_paged_fwd(dev[:, :8], *args, max_q=20)
    ref = R.attention(rows[:, :8].double(), *c.values(), c.table, c.start, c.kv_len, True, 1 / math.sqrt(128))
    check_attention(c, o.cpu(), lse.cpu(), ref)
    # heads first, and a token's heads far apart
    heads = rows[:, :8].transpose(0, 1).contiguous().cuda()
    o2, lse2 = M.attn_paged_fwd(heads.transpose(0, 1), *args, max_q=20)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_a_peaked_softmax_moves_its_reference():
    """Scores that grow along the keys by more than the reference may lag, and fall behind it by more than fp32's exponent."""
    from paper_2512_18134_amd import binding as M
    for dt in ("bf16", "f16"):
        c = Cache([1, 90], [600, 600], 1, 64, 16, dt, False, 16)
        for b in range(2):
            for p in range(600):
                page, at = R.place(c.table, c.n_pages, 16, b, p)
                c.pages[0][page, 0, at] = (0.25 * (p if b == 0 else 600 - p)) * torch.ones(64)
        q = torch.ones(91, 2, 64).to(R.DT[dt])
        _, o, lse, ref = attend(M, c, 2, True, 90, q)
        check_attention(c, o, lse, ref)


# ------------------------------------------------------------------------------------------------------- write and read

WRITES = [  # news, kvs, H_kv, D, page
    ([1], [1], 1, 64, 16),
    ([1] * 70, [3 * i + 1 for i in range(70)], 2, 128, 16),
    ([5, 0, 33, 1], [5, 9, 100, 64], 3, 256, 32),
    ([300, 2], [300, 513], 4, 64, 256),
    ([3, 2], [1, 2], 2, 128, 16),              # two rows lie before position 0
    ([1100, 1500], [1100, 1600], 2, 128, 64),  # enough rows for the wide variant
]


@pytest.mark.parametrize("shape", WRITES, ids=lambda s: "B%d_T%d_H%d_D%d_p%d" % (len(s[0]), sum(s[0]), *s[2:]))
@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
def test_rows_are_written_where_they_belong_and_read_back(shape, dt, e4m3):
    from paper_2512_18134_amd import binding as M
    news, kvs, H, D, page = shape
    c = Cache(news, kvs, H, D, page, dt, e4m3, 21, front=1, behind=2)
    k, v = c.rows(H), c.rows(H)
    k[-1 - 2] *= 1000                          # amplitudes of their own
    v *= torch.exp(torch.randn(c.T, H, 1, generator=c.gen)).to(v.dtype)
    v[:, 0] = 0                                # a row of zeros
    args, scales = c.on_gpu()
    before = [p.clone() for p in c.pages], [None if s is None else s.clone() for s in c.scale]
    out = fn(M, "attn_cache_write", dt)(k.cuda(), v.cuda(), *args, **scales)
    assert out[0] is args[0] and out[1] is args[1]
    want_rows = []
    for i, x in enumerate((k, v)):
        value, exponent = R.e4m3_row(x) if e4m3 else (x.double(), None)
        back = torch.full(x.shape, float("nan"), dtype=torch.float64)
        for b in range(len(news)):
            for r, p in enumerate(R.positions(c.start, c.kv_len, b)):
                t = int(c.start[b]) + r
                at = R.place(c.table, c.n_pages, page, b, p)
                back[t] = 0 if at is None else value[t]
                if at is None:
                    continue
                if e4m3:
                    before[1][i][at[0], :, at[1]] = (exponent[t] + 127).to(torch.uint8)
                    q = value[t] / torch.tensor(2.0, dtype=torch.float64) ** exponent[t][:, None]
                    before[0][i].view(torch.uint8)[at[0], :, at[1]] = q.float().to(torch.float8_e4m3fn).view(torch.uint8)
                else:
                    before[0][i][at[0], :, at[1]] = x[t]
        want_rows.append(back)
        pages = args[i].cpu()
        bits = torch.uint8 if e4m3 else torch.int16
        same = pages.view(bits) == before[0][i].view(bits)
        if e4m3:    # either zero
            same |= (pages.view(bits) & 0x7f == 0) & (before[0][i].view(bits) & 0x7f == 0)
            assert torch.equal(scales["kv"[i] + "_scale"].cpu(), before[1][i])
        assert same.all()
    nan = float("nan")
    given = [torch.full((H, c.T, D), nan, dtype=R.DT[dt], device="cuda").transpose(0, 1) for _ in "kv"]
    got = fn(M, "attn_cache_read", dt)(*args, c.T, **scales, k=given[0], v=given[1])
    again = fn(M, "attn_cache_read", dt)(*args, c.T, **scales)
    for g, a, w in zip(got, again, want_rows):
        g, mine = g.cpu(), ~torch.isnan(w)
        assert torch.equal(g[mine].double(), w.to(R.DT[dt])[mine].double())
        assert torch.isnan(g[~mine]).all()
        assert torch.equal(a.cpu()[mine], g[mine])


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_e4m3_rows_at_the_edges_of_their_units(dt):
    """Amplitudes at and next to 448 times a power of two, ties, subnormal elements, the type's largest and smallest."""
    from paper_2512_18134_amd import binding as M
    t, D = R.DT[dt], 64
    eps, big = torch.finfo(t).eps, torch.finfo(t).max
    rows = [torch.zeros(D) for _ in range(8)]
    rows[0][:4] = torch.tensor([448.0, 17.0, 18.0, 19.0])
    rows[1][:4] = torch.tensor([448.0 * (1 + eps), 1.0, -1.0625, 1.1875])
    rows[2][:6] = torch.tensor([1.0, 2.0 ** -8, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 2.0 ** -15])
    rows[3][:3] = torch.tensor([big, -big, big * 0.97])
    rows[4][:3] = torch.tensor([torch.finfo(t).smallest_normal, 2.0 ** -24, 1e-7])
    rows[5][:2] = torch.tensor([224.0, -0.4375])
    rows[6][:3] = torch.tensor([240.0, 248.0, -232.0]) * 2.0 ** -3
    x = torch.stack(rows).to(t)[:, None]
    pages = [torch.zeros(1, 1, 16, D).to(torch.float8_e4m3fn).cuda() for _ in "kv"]
    scale = [torch.zeros(1, 1, 16, dtype=torch.uint8, device="cuda") for _ in "kv"]
    index = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([[0]], [0, 8], [8])]
    fn(M, "attn_cache_write", dt)(x.cuda(), x.cuda(), *pages, *index, *scale)
    want, e = R.e4m3_row(x)
    assert torch.equal(R.cached(pages[0].cpu(), scale[0].cpu())[0, :, :8].transpose(0, 1), want)
    assert torch.equal(scale[0].cpu()[0, 0, :8].int() - 127, e[:, 0].int())
    k, v = fn(M, "attn_cache_read", dt)(*pages, *index, 8, *scale)
    assert torch.isfinite(k.float()).all() and torch.equal(k.cpu().double(), want.to(t).double()) and torch.equal(k, v)
    assert ((want - x.double()).abs() <= x.double().abs() * 2.0 ** -4 + 2.0 ** (e.double()[..., None] - 10)).all()


def test_rows_without_a_place_are_left_out():
    from paper_2512_18134_amd import binding as M
    c = Cache([40, 40], [200, 40], 2, 64, 16, "bf16", False, 31)
    c.table[0, 10] = c.n_pages
    c.table[0, 11] = -1
    c.kv_len[1] = -7
    args, _ = c.on_gpu()
    before = [p.clone() for p in args[:2]]
    k = c.rows(2).cuda()
    M.attn_cache_write(k, k, *args)
    back, _ = M.attn_cache_read(*args, c.T)
    ok = [R.place(c.table, c.n_pages, 16, 0, p) is not None for p in range(160, 200)]
    assert 0 < sum(ok) < 40
    for r in range(40):
        assert torch.equal(back[r], k[r] if ok[r] else torch.zeros_like(k[r]))
    assert (back[40:] == 0).all()
    changed = sum(int((a.view(torch.int16) != b.view(torch.int16)).any(-1).any(1).sum()) for a, b in zip(args[:2], before))
    assert changed == 2 * sum(ok)


def test_refusals():
    from paper_2512_18134_amd import binding as M
    c = Cache([2], [20], 2, 64, 16, "bf16", False, 41)
    args, _ = c.on_gpu()
    k, q = c.rows(2).cuda(), c.rows(4).cuda()
    with pytest.raises(TypeError):
        M.attn_cache_write_f16(k, k, *args)
    with pytest.raises(TypeError):
        M.attn_cache_write(k, k, *args, k_scale=torch.zeros(1), v_scale=torch.zeros(1))
    with pytest.raises(ValueError):
        M.attn_cache_write(k[:, :1], k[:, :1], *args)
    with pytest.raises(TypeError):
        M.attn_cache_write(k, k, *args[:2], args[2].long(), *args[3:])
    with pytest.raises(TypeError):
        M.attn_cache_write(k, k, *args[:3], args[3][:1], args[4])
    with pytest.raises(ValueError):
        M.attn_cache_read(*args, 2, k=k[:1].expand(2, 2, 64), v=k)
    with pytest.raises(ValueError):
        M.attn_paged_fwd(c.rows(3).cuda(), *args)
    with pytest.raises(ValueError):
        M.attn_paged_fwd(torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), *args)
    with pytest.raises(TypeError):
        M.attn_paged_fwd(q, *args, o=q[:1])
    for bad in (dict(scale=0.0), dict(max_q=0), dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(M.AttnError):
            M.attn_paged_fwd(q, *args, **bad)
    odd = [torch.zeros(3, 2, 48, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    with pytest.raises(M.AttnError):
        M.attn_paged_fwd(q, *odd, *args[2:])


def test_both_ways_of_the_binding_take_the_same_calls():
    """csrc/marshal.cpp for plain calls, Python for the rest: a `causal` or `interleaved` that is no bool, a scale or an int of
    another type sends a call the Python way."""
    from paper_2512_18134_amd import binding as M
    if M._native() is M._NotBuilt:
        pytest.skip("the extension module was left out of this build")
    same = lambda a, b: all(torch.equal(x, y) and x.dtype == y.dtype and x.shape == y.shape for x, y in zip(a, b))
    for dt, e4m3 in (("bf16", False), ("f16", True)):
        i = int(dt == "f16")
        c = Cache([3, 1, 40], [300, 64, 40], 2, 64, 16, dt, e4m3, 51)
        args, scales = c.on_gpu()
        s = (scales["k_scale"], scales["v_scale"])
        k, v, q = (c.rows(h).cuda() for h in (2, 2, 6))
        native = M._native()
        slow = lambda name, *a, **kw: getattr(M, name)(getattr(M._lib, "attn_" + kw.pop("entry") + ("_f16" if i else "")),
                                                       R.DT[dt], *a)
        before = [t.clone() for t in args[:2]]
        slow("_marshal_rows", k, v, *args, *s, None, entry="cache_write")
        one = [t.clone() for t in args[:2]]
        for t, b in zip(args[:2], before):
            t.copy_(b)
        assert native.write(i, k, v, *args, *s, None)[0] is args[0]
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(one, args[:2]))
        assert same(native.read(i, *args, c.T, *s, None, None, None), slow("_read", *args, c.T, *s, None, None, None,
                                                                           entry="cache_read"))
        for causal in (True, False):
            fast = native.paged(i, q, *args, *s, None, None, None, causal, None, 40, None)
            assert same(fast, slow("_marshal_paged", q, *args, *s, None, None, None, causal, None, 40, None, entry="paged_fwd"))
        rq, rk = q.transpose(0, 1)[None], k.transpose(0, 1)[None]
        pos = torch.arange(c.T, dtype=torch.int32, device="cuda")[None, None]
        freq = torch.rand(32, dtype=torch.float64, device="cuda")
        fast = native.rope(i, rq, rk, pos, freq, (32,), None, None, False, True, None)
        assert same(fast, slow("_marshal_rope", rq, rk, pos, freq, (32,), None, None, False, True, None, entry="rope"))
        # handed back: other types, overlapping outputs, another stream's allocation
        assert native.write(i, k.float(), v, *args, *s, None) is None
        assert native.read(i, *args, c.T, *s, k[:1].expand(c.T, 2, 64), v, None) is None
        assert native.paged(i, q, *args, *s, None, None, None, 1, None, 40, None) is None
        assert native.paged(i, q, *args, *s, None, None, None, True, None, None, torch.cuda.Stream()) is None
        assert native.rope(i, rq, None, pos, freq, (32,), None, None, False, True, None) is None
