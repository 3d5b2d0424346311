"""Chunks of many rows weighed, and what is chosen by them moved, in captured graphs: replayed with other rows, lengths and pages, and eager work between,
every replay against the same calls made eagerly on a copy of the state."""
import pytest
import torch

from test_eviction_serving_gpu import Pool, fn, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D, dt, e4m3, H, G, most", [(64, "f16", True, 2, 4, 1500), (64, "bf16", False, 1, 2, 1500), (128, "bf16", True, 2, 4, 1500),
                                                     (128, "f16", False, 8, 4, 9000), (256, "bf16", True, 2, 3, 1500), (256, "f16", False, 8, 4, 9000)])
def test_a_captured_chunk_is_weighed_and_cut(D, dt, e4m3, H, G, most):
    from paper_2512_18134_amd import binding as M
    B, n = 2, 96                                           # 192 rows and more of a key head: the kernel for many
    p = Pool(B, most, H, D, 16, dt, e4m3, 19)
    fill = p.rows(1000 * B, H).cuda()
    fn(M, "attn_cache_write", dt)(fill, fill, *p.pages, p.dev_table, i32([0, 1000, 2000]).cuda(), i32([1000] * B).cuda(), **p.scale)
    state = {"q": p.rows(B * n, H * G).cuda(), "lse": (torch.randn((B * n, H * G), generator=p.gen) + 6).cuda(), "table": p.dev_table.clone(),
             "start": i32([0, n, 2 * n]).cuda(), "kv": i32([1000] * B).cuda(), "seen": i32([1000] * B).cuda(), "keep": i32([900] * B).cuda(),
             "weights": torch.rand((B, H, p.L), generator=p.gen).cuda(),
             "stamps": torch.arange(p.L, dtype=torch.int32).expand(B, H, p.L).contiguous().cuda(),
             "k_pages": p.pages[0], "v_pages": p.pages[1], **p.scale}
    out = {"dst": torch.empty((B, H, 300), dtype=torch.int32, device="cuda"), "src": torch.empty((B, H, 300), dtype=torch.int32, device="cuda"),
           "new_len": torch.empty(B, dtype=torch.int32, device="cuda")}

    def step(s, o):
        fn(M, "attn_cache_weigh", dt)(s["q"], s["lse"], s["k_pages"], s["table"], s["start"], s["kv"], s["weights"], k_scale=s.get("k_scale"),
                                      stamps=s["stamps"], seen=s["seen"], decay=0.5, max_q=n)
        M.attn_cache_select(s["weights"], s["kv"], s["keep"], 300, s["stamps"], s["seen"], sinks=2, recent=40, **o)
        M.attn_cache_move(s["k_pages"], s["v_pages"], s["table"], o["dst"], o["src"], **{x: s[x] for x in p.scale}, weights=s["weights"],
                          stamps=s["stamps"])

    bits = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])
    clone = lambda d: {k: t.clone() for k, t in d.items()}
    first = clone(state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(state, out)
    for k in state:
        state[k].copy_(first[k])
    moved = 0
    for turn in range(4):
        state["q"].copy_(p.rows(B * n, H * G))
        state["lse"].copy_(torch.randn((B * n, H * G), generator=p.gen) + 6)
        kv = [1000 - 7 * turn, max(30, 250 * turn)]        # (the second one shorter than its rows at first)
        state["kv"].copy_(i32(kv)), state["seen"].copy_(i32([x + 60 * turn for x in kv]))
        state["keep"].copy_(i32([900 - 30 * turn, max(0, 200 * turn - 3)]))
        state["start"].copy_(i32([0, n - turn, 2 * n - turn]))
        if turn == 2:
            state["table"][0, 3] = -1
        eager, eager_out = clone(state), clone(out)
        graph.replay()
        torch.cuda.synchronize()
        step(eager, eager_out)
        torch.cuda.synchronize()
        for a, b in ((state, eager), (out, eager_out)):
            for k in a:
                assert torch.equal(bits(a[k]), bits(b[k])), (turn, k)
        moved += int((out["dst"] >= 0).sum())
    assert moved > 0
