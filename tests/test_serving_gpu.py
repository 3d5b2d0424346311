"""The serving operators together, as a model's layers call them: new tokens' queries and keys turned by their positions, keys
and values written into the paged cache, attention over it.  Prompts in chunks, decoding steps from captured graphs whose
lengths change between the replays, several streams, pools longer than 32-bit offsets."""
import math

import pytest
import torch

import serving_ref as R
from test_paged_gpu import Cache, check_attention, fn

pytestmark = pytest.mark.gpu

SECTIONS = (16, 24, 24)                      # three axes, D = 128


class Layer:
    """One attention layer's serving state: a cache that sequences grow into, static arrays for the step."""

    def __init__(self, M, dt, e4m3, lengths, T, H_kv=2, G=4, D=128, page=16, width=24, seed=61):
        self.M, self.dt, self.e4m3, self.H_kv, self.H_q, self.D, self.page = M, dt, e4m3, H_kv, H_kv * G, D, page
        self.gen = torch.Generator().manual_seed(seed)
        B = len(lengths)
        n_pages = B * width + 1
        ids = torch.randperm(n_pages, generator=self.gen)[:B * width].view(B, width).to(torch.int32)
        self.table, self.n_pages = ids, n_pages
        shape = (n_pages, H_kv, page, D)
        kind = torch.float8_e4m3fn if e4m3 else R.DT[dt]
        self.pages = [torch.zeros(shape, dtype=kind, device="cuda") for _ in "kv"]
        self.scales = [torch.zeros(shape[:3], dtype=torch.uint8, device="cuda") if e4m3 else None for _ in "kv"]
        self.lengths, self.T, self.B = list(lengths), T, B
        self.freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
        self.index = [ids.cuda(), torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
                      torch.zeros(B, dtype=torch.int32, device="cuda")]
        self.rows = torch.zeros(T, self.H_q + 2 * H_kv, D, dtype=R.DT[dt], device="cuda")
        self.pos = torch.zeros(3, 1, T, dtype=torch.int32, device="cuda")
        self.turned = [torch.zeros(T, h, D, dtype=R.DT[dt], device="cuda") for h in (self.H_q, H_kv)]
        self.o = torch.zeros(T, self.H_q, D, dtype=R.DT[dt], device="cuda")
        self.lse = torch.zeros(T, self.H_q, device="cuda")
        self.ws = torch.empty(M.attn_paged_fwd_workspace_bytes(T, B, self.H_q, H_kv, D), dtype=torch.uint8, device="cuda")

    def feed(self, news):
        """The next step's inputs, into the static arrays: news[b] new tokens of sequence b."""
        start = [sum(news[:b]) for b in range(self.B + 1)]
        self.lengths = [n + k for n, k in zip(news, self.lengths)]
        self.start, self.kv_len = (torch.tensor(x, dtype=torch.int32) for x in (start, self.lengths))
        pos = torch.zeros(3, 1, self.T, dtype=torch.int32)
        for b in range(self.B):
            p = torch.tensor(R.positions(self.start, self.kv_len, b), dtype=torch.int32)
            pos[0, 0, start[b]:start[b + 1]], pos[1, 0, start[b]:start[b + 1]] = p, p // 7
            pos[2, 0, start[b]:start[b + 1]] = p % 7
        self.host_rows = torch.randn(self.rows.shape, generator=self.gen).to(self.rows.dtype)
        self.rows.copy_(self.host_rows)
        self.pos.copy_(pos)
        self.index[1].copy_(self.start)
        self.index[2].copy_(self.kv_len)
        self.host_pos = pos

    def step(self, max_q, o=None, lse=None, ws=None, stream=None):
        M, H, Hk = self.M, self.H_q, self.H_kv
        heads = lambda x: x.transpose(0, 1)[None]
        q, k, v = self.rows[:, :H], self.rows[:, H:H + Hk], self.rows[:, H + Hk:]
        fn(M, "attn_rope", self.dt)(heads(q), heads(k), self.pos, self.freq, SECTIONS, *map(heads, self.turned), stream=stream)
        scales = dict(k_scale=self.scales[0], v_scale=self.scales[1], stream=stream)
        fn(M, "attn_cache_write", self.dt)(self.turned[1], v, *self.pages, *self.index, **scales)
        fn(M, "attn_paged_fwd", self.dt)(self.turned[0], *self.pages, *self.index, o=self.o if o is None else o,
                                         lse=self.lse if lse is None else lse, workspace=self.ws if ws is None else ws,
                                         max_q=max_q, **scales)

    def check(self):
        """Every stage against 64 bits, from what the stage before it has left (and the test before has checked)."""
        n, H, Hk = int(self.start[-1]), self.H_q, self.H_kv
        heads = lambda x: x.transpose(0, 1)[None]
        half = R.half_step(self.rows.dtype)
        for i, (a, b) in enumerate(((0, H), (H, H + Hk))):
            x = heads(self.host_rows[:, a:b])
            want = R.rope(x, self.host_pos, self.freq.cpu(), SECTIONS)
            got = heads(self.turned[i].cpu()).double()
            pair = torch.hypot(x.double()[..., :64], x.double()[..., 64:]).repeat(1, 1, 1, 2)
            # the product's rounding, and three of fp32 with an angle reduced to 2^-24 of a turn
            bound = half * want.abs() * (1 + half) + pair * 2.0 ** -20 + (2.0 ** -25 if self.dt == "f16" else 0)
            assert ((got - want).abs() <= bound).all()
        for i, x in enumerate((self.turned[1].cpu(), self.host_rows[:, H + Hk:])):
            value, exponent = R.e4m3_row(x) if self.e4m3 else (x.double(), None)
            pool = R.cached(self.pages[i].cpu(), None if not self.e4m3 else self.scales[i].cpu())
            for b in range(self.B):
                for r, p in enumerate(R.positions(self.start, self.kv_len, b)):
                    page, at = R.place(self.table, self.n_pages, self.page, b, p)
                    assert torch.equal(pool[page, :, at], value[int(self.start[b]) + r])
        pools = [R.cached(p.cpu(), s if s is None else s.cpu()) for p, s in zip(self.pages, self.scales)]
        ref = R.attention(self.turned[0].cpu().double(), *pools, self.table, self.start, self.kv_len, True, self.D ** -0.5)
        o, lse = self.o.cpu().clone(), self.lse.cpu().clone()
        o[n:], lse[n:] = float("nan"), float("nan")        # the static rows behind the last token
        check_attention(self, o, lse, ref)


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
def test_prompts_in_chunks_and_then_steps(dt, e4m3):
    from paper_2512_18134_amd import binding as M
    s = Layer(M, dt, e4m3, [0, 0, 0], 200)
    for news in ([150, 0, 7], [30, 60, 90], [1, 1, 1], [4, 0, 1], [1, 1, 0]):
        s.feed(news)
        s.step(max(news))
        s.check()


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("bf16", True), ("f16", False)])
def test_a_captured_step_follows_the_lengths(dt, e4m3):
    from paper_2512_18134_amd import binding as M
    s = Layer(M, dt, e4m3, [0, 0, 0, 0], 200)
    s.feed([90, 5, 0, 33])
    s.step(90)
    # two layers' steps with one workspace, in two graphs
    t = Layer(M, dt, e4m3, [0, 0, 0, 0], 4, seed=62)
    s.T = t.T = 4
    s.rows, s.pos, s.turned, s.o, s.lse = t.rows.clone(), t.pos.clone(), [x.clone() for x in t.turned], t.o.clone(), t.lse.clone()
    s.feed([1, 1, 1, 1]), t.feed([1, 1, 1, 1])
    t.ws = s.ws
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for x in (s, t):
            x.step(1)
    torch.cuda.current_stream().wait_stream(side)
    for x in (s, t):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.step(1)
    own = torch.empty_like(s.ws)
    for news in ([1, 1, 1, 1], [1, 0, 1, 1], [0, 0, 0, 0], [1, 1, 0, 0], [1, 1, 1, 1]):
        for x, g in ((s, graphs[0]), (t, graphs[1])):
            x.feed(news)
            g.replay()
            torch.cuda.synchronize()
            pools = [p.clone() for p in x.pages]
            o, lse = x.o.clone(), x.lse.clone()
            x.step(1, o2 := torch.zeros_like(o), lse2 := torch.zeros_like(lse), own)      # again, eagerly
            n = sum(news)
            assert torch.equal(o[:n], o2[:n]) and torch.equal(lse[:n], lse2[:n])
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(pools, x.pages))
            x.check()


def test_other_streams():
    from paper_2512_18134_amd import binding as M
    s = Layer(M, "bf16", False, [0, 0], 100)
    s.feed([70, 30])
    s.step(70)
    torch.cuda.synchronize()
    o, lse = s.o.clone(), s.lse.clone()
    for how in ("argument", "current"):
        s.o.zero_(), s.lse.zero_(), s.pages[0].zero_(), s.pages[1].zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        if how == "argument":
            s.step(70, stream=side)
        else:
            with torch.cuda.stream(side):
                s.step(70)
        side.synchronize()
        assert torch.equal(s.o, o) and torch.equal(s.lse, lse)
    # outputs and workspace of the call's own
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = M.attn_paged_fwd(s.turned[0], *s.pages, *s.index, max_q=70, stream=side)
        side.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse)


def test_two_calls_at_once():
    from paper_2512_18134_amd import binding as M
    layers = [Layer(M, "bf16", False, [0] * 3, 300, seed=71, width=12), Layer(M, "bf16", True, [0] * 4, 8, G=8, seed=72),
              Layer(M, "f16", False, [0] * 2, 40, seed=73)]
    for s, news in zip(layers, ([190, 9, 100], [2, 2, 2, 2], [1, 39])):
        s.feed(news)
        s.max_q = max(news)
        s.step(s.max_q)
    torch.cuda.synchronize()
    want = [(s.o.clone(), s.lse.clone()) for s in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for s in layers:
            s.o.zero_(), s.lse.zero_()
        torch.cuda.synchronize()
        for _ in range(4):
            for s, stream in zip(layers, streams):
                s.step(s.max_q, stream=stream)
        torch.cuda.synchronize()
        for s, (o, lse) in zip(layers, want):
            assert torch.equal(s.o, o) and torch.equal(s.lse, lse)


@pytest.mark.parametrize("n, e4m3", [(1, False), (1, True), (90, False), (90, True)])
def test_pages_far_behind_the_pools_start(n, e4m3):
    """Pools of more than 2^32 elements; only the pages in use are written or read."""
    from paper_2512_18134_amd import binding as M
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    H, D, page = 8, 128, 256
    n_pages = (2 ** 32 + 2 ** 31) // (H * page * D)
    kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    big = [torch.empty((n_pages, H, page, D), dtype=kind, device="cuda") for _ in "kv"]
    scales = [torch.empty((n_pages, H, page), dtype=torch.uint8, device="cuda") if e4m3 else None for _ in "kv"]
    gen = torch.Generator().manual_seed(81)
    kv = 700
    k, v = (torch.randn(kv, H, D, generator=gen).bfloat16() for _ in "kv")
    q = torch.randn(n, 2 * H, D, generator=gen).bfloat16()
    ids = [n_pages - 1, 5, n_pages - 3]
    index = lambda rows: [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([ids], [0, rows], [kv])]
    M.attn_cache_write(k.cuda(), v.cuda(), *big, *index(kv), *scales)
    back = M.attn_cache_read(*big, *index(kv), kv, *scales)
    want = [R.e4m3_row(x)[0] if e4m3 else x.double() for x in (k, v)]
    for g, w in zip(back, want):
        assert torch.equal(g.cpu().double(), w.bfloat16().double())
    o, lse = M.attn_paged_fwd(q.cuda(), *big, *index(n), *scales, max_q=n)
    small = [torch.zeros(3, H, page, D, dtype=torch.float64) for _ in "kv"]
    for s, w in zip(small, want):
        for p in range(kv):
            s[p // page, :, p % page] = w[p]
    c = Cache([n], [kv], H, D, page, "bf16", False, 82)
    ref = R.attention(q.double(), *small, torch.tensor([[0, 1, 2]], dtype=torch.int32), c.start, c.kv_len, True, D ** -0.5)
    check_attention(c, o.cpu(), lse.cpu(), ref)


@pytest.mark.parametrize("extra", [(), ("--serve-cache", "e4m3", "--serve-new", "3", "--dtype", "f16")], ids=["bf16", "f16_e4m3"])
def test_bench_line_of_a_decoding_step(extra):
    from test_bench_tools_gpu import run_bench
    d = run_bench("--serve", "8", "--serve-context", "2000", "--steps", "5", "--warmup", "2", *extra)
    for key in ("metric", "value", "unit", "n_gpus", "steps", "warmup", "ms_per_step", "higher_is_better", "scaling",
                "vs_baseline", "dtype", "data", "config", "roofline"):
        assert key in d, key
    assert d["value"] > 0 and d["steps"] == 5 and 0 < d["roofline"]["frac"] < 1
