"""Captured steps of the larger kinds: chunks of prompts next to decoding sequences (two attention kernels and the merge), a batch of
more sequences than work their cut out themselves, rows written and read in runs, rotary positions of many tokens.  Every replay,
with lengths, pages and rows of its own and the program's eager work between them, has the bits of the eager call."""
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


class Step:
    def __init__(self, M, B, T, H_kv, G, D, page, width, dt, e4m3, max_q, seed):
        self.M, self.B, self.T, self.max_q, self.e4m3, self.suffix = M, B, T, max_q, e4m3, "_f16" if dt == "f16" else ""
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)
        self.page, self.width, self.n_pages = page, width, B * width + 5
        empty = lambda *s, dtype=R.DT[dt]: torch.zeros(s, dtype=dtype, device="cuda")
        self.q, self.k, self.v = empty(T, H_kv * G, D), empty(T, H_kv, D), empty(T, H_kv, D)
        self.pages = [empty(self.n_pages, H_kv, page, D, dtype=torch.float8_e4m3fn if e4m3 else R.DT[dt]) for _ in "kv"]
        self.scale = [empty(self.n_pages, H_kv, page, dtype=torch.uint8) if e4m3 else None for _ in "kv"]
        self.table, self.start, self.kv_len = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B, width), (B + 1,), (B,)))
        self.pos = torch.zeros(1, 1, T, dtype=torch.int32, device="cuda")
        self.freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") / (D // 2))
        self.ws = torch.empty(M.attn_paged_fwd_workspace_bytes(T, B, H_kv * G, H_kv, D), dtype=torch.uint8, device="cuda")
        self.D = D

    def outputs(self):
        return [torch.full_like(x, 7) for x in (self.q, self.k, self.q, self.k, self.v)] + [torch.full(self.q.shape[:2], 7.0, device="cuda")]

    def feed(self, news, kvs):
        """News and lengths, new pages and rows, and the pool as it is before the step."""
        assert len(news) == self.B and sum(news) <= self.T and max(kvs) <= self.page * self.width
        self.table.copy_(torch.randperm(self.n_pages, generator=self.host)[:self.B * self.width].view(self.B, self.width).int())
        self.table[1, 0] = -1
        self.start.copy_(torch.tensor([sum(news[:b]) for b in range(self.B + 1)], dtype=torch.int32))
        self.kv_len.copy_(torch.tensor(kvs, dtype=torch.int32))
        for x in (self.q, self.k, self.v):
            x.normal_(generator=self.gen)
        for p in self.pages:
            if self.e4m3:
                p.view(torch.uint8).random_(0, 0x70, generator=self.gen)
            else:
                p.normal_(generator=self.gen)
        for s in self.scale:
            if s is not None:
                s.random_(117, 121, generator=self.gen)
        self.pos.random_(0, 100000, generator=self.gen)
        self.before = [p.clone() for p in self.pages], [s if s is None else s.clone() for s in self.scale]

    def again(self):
        for p, b in zip(self.pages, self.before[0]):
            p.copy_(b)
        for s, b in zip(self.scale, self.before[1]):
            if s is not None:
                s.copy_(b)

    def run(self, out, ws):
        call = lambda name: getattr(self.M, name + self.suffix)
        heads = lambda x: x.transpose(0, 1)[None]
        cache = (*self.pages, self.table, self.start, self.kv_len)
        call("attn_rope")(heads(self.q), heads(self.k), self.pos, self.freq, (self.D // 2,), heads(out[0]), heads(out[1]))
        call("attn_cache_write")(out[1], self.v, *cache, *self.scale)
        call("attn_paged_fwd")(out[0], *cache, *self.scale, o=out[2], lse=out[5], workspace=ws, max_q=self.max_q)
        call("attn_cache_read")(*cache, self.T, *self.scale, k=out[3], v=out[4])


CASES = [  # B, T, H_kv, G, D, page, width, dt, e4m3, max_q, [(news, kvs)]
    (6, 4200, 4, 4, 128, 16, 200, "bf16", False, 2000,
     [([2000, 1, 1, 700, 0, 1], [3100, 900, 1, 700, 50, 3000]), ([1, 1, 900, 1, 1, 2000], [3101, 901, 3200, 701, 51, 2000]),
      ([1] * 6, [3102, 902, 1, 702, 52, 2001]), ([0] * 6, [5] * 6)]),
    (5, 4300, 4, 2, 64, 32, 130, "f16", True, 1500, [([1500, 2, 0, 1, 1200], [4000, 500, 9, 4100, 1200]), ([1, 1, 1500, 1, 1], [4001, 501, 1600, 4101, 1201]),
                                                     ([300, 3, 5, 0, 1], [4160, 504, 1605, 4101, 1202])]),
    (200, 4100, 4, 4, 128, 16, 40, "bf16", True, 300, [([300] + [1] * 199, [640 - i % 500 for i in range(200)]),
                                                       ([1] * 100 + [0] * 99 + [250], [639 - i % 300 for i in range(200)])]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "B%d_D%d_%s%s" % (c[0], c[4], c[7], "_e4m3" if c[8] else ""))
def test_replays_have_the_bits_of_eager_calls(case):
    from paper_2512_18134_amd import binding as M
    steps = [Step(M, *case[:10], seed) for seed in (41, 42)]
    one, two = steps
    two.ws = one.ws                                        # two graphs that share a workspace and run one behind the other
    outs, graphs = [s.outputs() for s in steps], []
    for s, out in zip(steps, outs):
        s.feed(*case[10][0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.run(out, s.ws)
        torch.cuda.current_stream().wait_stream(side)
        s.again()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.run(out, s.ws)
    own = torch.empty_like(one.ws)
    for news, kvs in case[10] + case[10][::-1]:
        for s, out, graph in zip(steps, outs, graphs):
            s.feed(news, kvs)
            for x in out:
                x.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            after = [p.clone() for p in s.pages]
            s.again()
            eager = s.outputs()
            s.run(eager, own)
            raw = lambda x: x.view(torch.uint8)
            assert all(torch.equal(raw(a), raw(b)) for a, b in zip(out, eager))
            assert all(torch.equal(raw(a), raw(b)) for a, b in zip(after, s.pages))
            n = sum(news)
            assert (eager[2][n:] == 7).all() and (eager[5][n:] == 7).all() and torch.isfinite(eager[2].float()).all()
