"""Trees of drafts, accumulated weights and eviction as a serving program runs them: one after the other over the same cache, in captured
graphs whose lengths change, on another stream, and by both of the binding's ways to the library."""
import math

import pytest
import torch

import evict_ref as E
import serving_ref as R
import tree_ref as T
from test_paged_gpu import check_attention, fn

pytestmark = pytest.mark.gpu


class Pool:
    """A cache of B sequences with room for `most` positions each, filled through attn_cache_write."""

    def __init__(self, B, most, H_kv, D, page, dt, e4m3, seed):
        self.gen = torch.Generator().manual_seed(seed)
        self.dt, self.e4m3, self.H_kv, self.D, self.page, self.B = dt, e4m3, H_kv, D, page, B
        width = -(-most // page)
        self.n_pages = B * width + 2
        self.table = torch.randperm(self.n_pages, generator=self.gen)[:B * width].view(B, width).to(torch.int32)
        shape = (self.n_pages, H_kv, page, D)
        if e4m3:
            self.pages = [torch.zeros(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in "kv"]
            self.scale = dict(zip(("k_scale", "v_scale"), (torch.full(shape[:3], 127, dtype=torch.uint8, device="cuda") for _ in "kv")))
        else:
            self.pages = [torch.zeros(shape, dtype=R.DT[dt], device="cuda") for _ in "kv"]
            self.scale = {}
        self.dev_table = self.table.cuda()
        self.L = width * page

    def rows(self, T, H):
        return torch.randn((T, H, self.D), generator=self.gen).to(R.DT[self.dt])

    def values(self):
        scales = [s.cpu() for s in self.scale.values()] or [None, None]
        return [R.cached(p.cpu(), s) for p, s in zip(self.pages, scales)]


i32 = lambda x: torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", True)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_verified_tree_leaves_the_sequence_that_was_accepted(D, dt, e4m3):
    """Drafts are written and attended to, the accepted path moves up, and the next token attends to what a sequence without drafts would
    have: the prefix and the accepted tokens in their order."""
    from paper_2512_18134_amd import binding as M
    H, G, kvs, n = 2, 4, [37, 300], [12, 20]
    p = Pool(2, 352, H, D, 16, dt, e4m3, 3)
    total = [a + b for a, b in zip(kvs, n)]
    k, v = p.rows(sum(total), H), p.rows(sum(total), H)
    start = i32([0, total[0], sum(total)])
    fn(M, "attn_cache_write", dt)(k.cuda(), v.cuda(), *p.pages, p.dev_table, start.cuda(), i32(total).cuda(), **p.scale)
    sets = [T.random_tree(m, 5 + b) for b, m in enumerate(n)]
    start = i32([0, n[0], sum(n)])
    q = p.rows(sum(n), H * G)
    mask = T.mask_tensor(sum(n), start, sets, 1)
    o, lse = fn(M, "attn_paged_tree", dt)(q.cuda(), *p.pages, p.dev_table, start.cuda(), i32(total).cuda(), mask.cuda(), **p.scale, max_q=20)
    ref = T.attention(q.double(), *p.values(), p.table, start, i32(total), mask, 1 / math.sqrt(D))

    class C:
        pass
    c = C()
    c.dt, c.kv_len = dt, i32(total)
    check_attention(c, o.cpu(), lse.cpu(), ref)
    # the deepest path of each tree
    dst, src, left = torch.full((2, 1, 20), -1, dtype=torch.int32), torch.full((2, 1, 20), -1, dtype=torch.int32), []
    paths = []
    for b in range(2):
        best = max(sets[b], key=lambda bits: bin(bits).count("1"))
        path = [i for i in range(n[b]) if best >> i & 1]
        dst[b, 0, :len(path)] = kvs[b] + torch.arange(len(path))
        src[b, 0, :len(path)] = kvs[b] + torch.tensor(path)
        paths.append(path)
        left.append(kvs[b] + len(path))
    before = p.values()
    M.attn_cache_move(*p.pages, p.dev_table, dst.cuda(), src.cuda(), **p.scale)
    after = p.values()
    for b in range(2):
        places = list(range(kvs[b])) + [kvs[b] + i for i in paths[b]]
        for old, new in zip(before, after):
            for to, come in enumerate(places):
                x, y = R.place(p.table, p.n_pages, 16, b, to), R.place(p.table, p.n_pages, 16, b, come)
                assert torch.equal(new[x[0], :, x[1]], old[y[0], :, y[1]])
    q = p.rows(2, H * G)
    start = i32([0, 1, 2])
    o, lse = fn(M, "attn_paged_fwd", dt)(q.cuda(), *p.pages, p.dev_table, start.cuda(), i32(left).cuda(), **p.scale, max_q=1)
    c.kv_len = i32(left)
    check_attention(c, o.cpu(), lse.cpu(), R.attention(q.double(), *after, p.table, start, i32(left), True, 1 / math.sqrt(D)))


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("bf16", True)])
def test_steps_with_evictions_keep_what_the_formulas_keep(dt, e4m3):
    """A prompt and decoding steps are weighed; whenever a sequence is 8 places over its budget it is cut.  The state beside the cache is
    checked against the plain implementations at every step, from the state before it."""
    from paper_2512_18134_amd import binding as M
    H, G, D, B = 2, 2, 64, 2
    p = Pool(B, 128, H, D, 16, dt, e4m3, 7)
    scale = 1 / math.sqrt(D)
    weights = torch.zeros((B, H, p.L), device="cuda")
    stamps = torch.zeros((B, H, p.L), dtype=torch.int32, device="cuda")
    kv, seen, budget = i32([0, 0]), i32([0, 0]), i32([40, 100])
    cuts = 0
    for step, n in enumerate([[60, 30]] + [[1, 1]] * 6 + [[3, 2]] * 20):
        kv, seen = kv + i32(n), seen + i32(n)
        start = i32([0, n[0], sum(n)])
        k, v, q = p.rows(sum(n), H), p.rows(sum(n), H), p.rows(sum(n), H * G)
        index = p.dev_table, start.cuda(), kv.cuda()
        fn(M, "attn_cache_write", dt)(k.cuda(), v.cuda(), *p.pages, *index, **p.scale)
        o, lse = fn(M, "attn_paged_fwd", dt)(q.cuda(), *p.pages, *index, **p.scale, max_q=max(n))
        old_w, old_s = weights.cpu(), stamps.cpu()
        fn(M, "attn_cache_weigh", dt)(q.cuda(), lse, p.pages[0], *index, weights, k_scale=p.scale.get("k_scale"), stamps=stamps,
                                      seen=seen.cuda(), decay=0.9, max_q=max(n))
        want, bound, want_s = E.weigh(q.double(), lse.cpu(), p.values()[0], p.table, start, kv, old_w, float(torch.tensor(0.9)), True, scale,
                                      old_s, seen)
        assert torch.equal(stamps.cpu(), want_s)
        assert ((weights.cpu().double() - want).abs() <= bound + 1e-30).all()
        over = kv >= budget + 8
        if not over.any():
            continue
        cuts += 1
        keep = torch.where(over, budget, kv)
        args = (weights.cpu(), kv, keep, 64, stamps.cpu(), seen)
        dst, src, new_len = M.attn_cache_select(weights, kv.cuda(), keep.cuda(), 64, stamps, seen.cuda(), sinks=2, recent=6)
        for g, w in zip((dst, src, new_len), E.select(*args, sinks=2, recent=6)):
            assert torch.equal(g.cpu(), w)
        before = [t.cpu() for t in (*p.pages, *p.scale.values())]
        rows = [weights.cpu(), stamps.cpu()]
        M.attn_cache_move(*p.pages, p.dev_table, dst, src, **p.scale, weights=weights, stamps=stamps)
        E.move(before, rows, p.table, 16, dst.cpu(), src.cpu())
        as_int = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16)
        for g, w in zip((*p.pages, *p.scale.values()), before):
            assert torch.equal(as_int(g.cpu()), as_int(w))
        assert torch.equal(weights.cpu(), rows[0]) and torch.equal(stamps.cpu(), rows[1])
        kv = new_len.cpu()
        for b in range(B):                                 # the first two and the last six tokens are there
            if over[b]:
                for h in range(H):
                    have = set(stamps[b, h, :int(kv[b])].tolist())
                    assert {0, 1} | set(range(int(seen[b]) - 6, int(seen[b]))) <= have
    assert cuts >= 3


def test_a_captured_step_is_replayed_as_lengths_and_masks_change():
    """Write, tree, weigh, select (in both of its ways) and move in one graph, replayed with eager work between: every replay against the same calls
    made eagerly on a copy of the state."""
    from paper_2512_18134_amd import binding as M
    H, G, D, B, n = 2, 4, 128, 3, 8
    for most in (400, 9000):
        p = Pool(B, most, H, D, 16, "bf16", False, 11)
        T_rows = B * n
        fill = p.rows(300 * B, H)
        M.attn_cache_write(fill.cuda(), fill.cuda(), *p.pages, p.dev_table, i32([0, 300, 600, 900]).cuda(), i32([300] * B).cuda())
        state = {"k": p.rows(T_rows, H).cuda(), "v": p.rows(T_rows, H).cuda(), "q": p.rows(T_rows, H * G).cuda(),
                 "start": i32([0, n, 2 * n, 3 * n]).cuda(), "kv": i32([308] * B).cuda(), "seen": i32([308] * B).cuda(),
                 "keep": i32([300] * B).cuda(), "mask": T.mask_tensor(T_rows, [0, n, 2 * n], [T.random_tree(n, b) for b in range(B)], 1).cuda(),
                 "weights": torch.rand((B, H, p.L), generator=p.gen).cuda(), "stamps": torch.arange(p.L, dtype=torch.int32).expand(B, H, p.L).contiguous().cuda(),
                 "k_pages": p.pages[0], "v_pages": p.pages[1]}
        out = {"o": torch.empty((T_rows, H * G, D), dtype=torch.bfloat16, device="cuda"), "lse": torch.empty((T_rows, H * G), device="cuda"),
               "dst": torch.empty((B, H, 16), dtype=torch.int32, device="cuda"), "src": torch.empty((B, H, 16), dtype=torch.int32, device="cuda"),
               "new_len": torch.empty(B, dtype=torch.int32, device="cuda")}
        ws = torch.empty(M.attn_paged_tree_workspace_bytes(T_rows, B, H * G, H, D), dtype=torch.uint8, device="cuda")
        ws2 = torch.empty(max(16, M.attn_cache_select_workspace_bytes(B, H, p.L)), dtype=torch.uint8, device="cuda")

        def step(s, o, ws, ws2):
            index = p.dev_table, s["start"], s["kv"]
            M.attn_cache_write(s["k"], s["v"], s["k_pages"], s["v_pages"], *index)
            M.attn_paged_tree(s["q"], s["k_pages"], s["v_pages"], *index, s["mask"], o=o["o"], lse=o["lse"], workspace=ws, max_q=n)
            M.attn_cache_weigh(s["q"], o["lse"], s["k_pages"], *index, s["weights"], stamps=s["stamps"], seen=s["seen"], decay=0.5, max_q=n)
            M.attn_cache_select(s["weights"], s["kv"], s["keep"], 16, s["stamps"], s["seen"], sinks=2, recent=n, dst=o["dst"], src=o["src"],
                                new_len=o["new_len"], workspace=ws2)
            M.attn_cache_move(s["k_pages"], s["v_pages"], p.dev_table, o["dst"], o["src"], weights=s["weights"], stamps=s["stamps"])

        clone = lambda d: {k: t.clone() for k, t in d.items()}
        start_state = clone(state)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(state, out, ws, ws2)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(state, out, ws, ws2)
        for k in state:
            state[k].copy_(start_state[k])
        for turn in range(5):
            for name in ("k", "v", "q"):
                state[name].copy_(p.rows(T_rows, state[name].shape[1]))
            lens = [300 + n, max(n, 40 * turn), 308 - turn]
            state["kv"].copy_(i32(lens)), state["seen"].copy_(i32([x + 100 * turn for x in lens]))
            state["keep"].copy_(i32([300, max(0, 40 * turn - 5), 300 - 2 * turn]))
            state["mask"].copy_(T.mask_tensor(T_rows, [0, n, 2 * n], [T.random_tree(n, 10 * turn + b) for b in range(B)], 1))
            ws.fill_(0xff), ws2.fill_(0xff)
            eager, eager_out = clone(state), clone(out)
            graph.replay()
            torch.cuda.synchronize()
            step(eager, eager_out, ws.clone(), ws2.clone())
            torch.cuda.synchronize()
            for a, b in ((state, eager), (out, eager_out)):
                for k in a:
                    x, y = (t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in (a[k], b[k]))
                    assert torch.equal(x.nan_to_num(3.0) if x.is_floating_point() else x, y.nan_to_num(3.0) if y.is_floating_point() else y), (turn, k)
            assert out["dst"].max() >= 0


def test_both_ways_give_the_same_and_refuse_the_same():
    """The extension module and the Python marshalling: a numpy-like number, an int decay or a stream object that is no plain one sends a call the
    other way."""
    from paper_2512_18134_amd import binding as M
    p = Pool(2, 128, 2, 64, 16, "bf16", False, 13)
    kv, start = i32([100, 50]).cuda(), i32([0, 3, 8]).cuda()
    rows = p.rows(150, 2).cuda()
    M.attn_cache_write(rows, rows, *p.pages, p.dev_table, i32([0, 100, 150]).cuda(), kv)
    q = p.rows(8, 4).cuda()
    mask = torch.full((8, 1), -1, dtype=torch.int64, device="cuda")

    class Number(int):
        pass
    index = p.dev_table, start, kv
    a, b = (M.attn_paged_tree(q, *p.pages, *index, mask, max_q=m) for m in (5, Number(5)))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    w = [torch.zeros((2, 2, p.L), device="cuda") for _ in range(2)]
    for x, decay in zip(w, (1.0, 1)):
        assert M.attn_cache_weigh(q, a[1], p.pages[0], *index, x, decay=decay) is x
    assert torch.equal(*w)
    keep = i32([60, 20]).cuda()
    a, b = (M.attn_cache_select(w[0], kv, keep, m) for m in (40, Number(40)))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = M.attn_cache_select(w[0], kv, keep, 40, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, c))
    bad = [
        (TypeError, lambda n: M.attn_paged_tree(q, *p.pages, *index, mask.int(), max_q=n)),
        (TypeError, lambda n: M.attn_paged_tree(q, *p.pages, *index, mask[:7], max_q=n)),
        (TypeError, lambda n: M.attn_paged_tree(q, *p.pages, *index, mask.t(), max_q=n)),
        (TypeError, lambda n: M.attn_paged_tree(q, *p.pages, *index, mask.cpu(), max_q=n)),
        (M.AttnError, lambda n: M.attn_paged_tree(q, *p.pages, *index, mask, scale=0.0, max_q=n)),
        (TypeError, lambda n: M.attn_cache_weigh(q, w[0], p.pages[0], *index, w[0], max_q=n)),
        (TypeError, lambda n: M.attn_cache_weigh(q, a[2].float(), p.pages[0], *index, None, max_q=n)),
        (TypeError, lambda n: M.attn_cache_weigh(q, torch.zeros(8, 4, device="cuda"), p.pages[0], *index, w[0], stamps=a[0], max_q=n)),
        (M.AttnError, lambda n: M.attn_cache_weigh(q, torch.zeros(8, 4, device="cuda"), p.pages[0], *index, w[0], decay=-1.0, max_q=n)),
        (TypeError, lambda n: M.attn_cache_select(w[0].double(), kv, keep, n)),
        (TypeError, lambda n: M.attn_cache_select(w[0], kv[:1], keep, n)),
        (M.AttnError, lambda n: M.attn_cache_select(w[0], kv, keep, n, new_len=kv)),
        (M.AttnError, lambda n: M.attn_cache_select(w[0], kv, keep, n, sinks=type(n)(2) - 3)),
    ]
    for error, call in bad:
        for number in (int, Number):
            with pytest.raises((error, ValueError)):
                call(number(5))
    dst, src = a[:2]
    for call in (lambda: M.attn_cache_move(*p.pages, p.dev_table, dst, src[:, :1].contiguous()), lambda: M.attn_cache_move(*p.pages, p.dev_table[:1], dst, src),
                 lambda: M.attn_cache_move(*p.pages, p.dev_table, dst.long(), src), lambda: M.attn_cache_move(*p.pages, p.dev_table, dst, src, weights=w[0][:1]),
                 lambda: M.attn_cache_move(p.pages[0].float(), p.pages[1], p.dev_table, dst, src)):
        with pytest.raises((TypeError, ValueError)):
            call()
