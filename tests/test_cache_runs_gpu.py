"""Writing and reading the paged cache in runs of eight tokens, which calls with enough rows take (csrc/attn_cache.hip): whose a
token is among many empty sequences, places without a page, rows of nobody, odd counts of tokens and heads, pools beyond 2^32
elements.  test_serving_launches.py holds these sizes to the kernel that they are for."""
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu

SIZES = [  # D, H_kv, T, page: enough waves for runs; T no multiple of 8, heads that end inside a wave's last slice
    (64, 5, 4099, 16),
    (64, 1, 8195, 256),
    (128, 3, 4101, 32),
    (128, 2, 8197, 16),
    (256, 3, 2733, 64),
    (256, 1, 8199, 128),
]


def batch(T, page, seed):
    """(news, kvs, front, behind): more than 64 empty sequences inside one run of eight tokens, single tokens, a long prompt."""
    gen = torch.Generator().manual_seed(seed)
    pick = lambda lo, hi: int(torch.randint(lo, hi, (1,), generator=gen))
    news = [3] + [0] * 70 + [2] + [0] * 130 + [1, 0, 1] + [1] * 60 + [0] * 64 + [9, 0, 0, 17, 400]
    front, behind = 5, 11
    news.append(T - front - behind - sum(news))
    kvs = [n + pick(0, 3 * page) for n in news]
    kvs[0] = 1                                             # two of its three rows lie in front of position 0
    kvs[1] = 0
    kvs[-2] = news[-2] - 7                                 # seven
    return news, kvs, front, behind


class Rows:
    def __init__(self, D, H, T, page, dt, e4m3, n_pages=0, seed=91):
        gen = torch.Generator().manual_seed(seed)
        self.D, self.H, self.T, self.page, self.dt, self.e4m3 = D, H, T, page, dt, e4m3
        self.news, self.kvs, front, behind = batch(T, page, seed)
        need = [-(-kv // page) for kv in self.kvs]
        self.n_pages = max(n_pages, sum(need) + 3)
        # (of a large pool its last pages)
        ids = (self.n_pages - 1 - torch.randperm(sum(need) + 3, generator=gen)[:sum(need)]).int()
        self.table = torch.full((len(self.news), max(need) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        wide = need.index(max(need))
        self.table[wide, 1], self.table[wide, 3], self.table[wide, need[wide] - 1] = -1, self.n_pages, 2 ** 31 - 1
        self.start = torch.tensor([front + sum(self.news[:b]) for b in range(len(self.news) + 1)], dtype=torch.int32)
        self.kv_len = torch.tensor(self.kvs, dtype=torch.int32)
        # every token's page (-1: it has no place) and place; whose == -1: nobody's
        seq = torch.repeat_interleave(torch.arange(len(self.news)), torch.tensor(self.news))
        whose = torch.full((T,), -1)
        whose[front:T - behind] = seq
        i = torch.arange(T) - self.start.long()[whose.clamp(min=0)]
        news, kvs = torch.tensor(self.news), torch.tensor(self.kvs)
        pos = (kvs - news)[whose.clamp(min=0)] + i
        page_of = self.table[whose.clamp(min=0), (pos // page).clamp(0, self.table.shape[1] - 1)].long()
        there = (whose >= 0) & (pos >= 0) & (page_of >= 0) & (page_of < self.n_pages)
        self.mine, self.there = whose >= 0, there
        self.page_of, self.place = page_of[there], (pos % page)[there]
        rows = lambda: torch.randn((T, H, D), generator=gen) * torch.exp(2 * torch.randn((T, H, 1), generator=gen))
        self.k, self.v = rows().to(R.DT[dt]), rows().to(R.DT[dt])
        shape = (self.n_pages, H, page, D)
        self.pages = [torch.empty(shape, dtype=torch.float8_e4m3fn if e4m3 else R.DT[dt], device="cuda") for _ in "kv"]
        self.scale = [torch.empty(shape[:3], dtype=torch.uint8, device="cuda") if e4m3 else None for _ in "kv"]
        self.index = [t.cuda() for t in (self.table, self.start, self.kv_len)]

    def call(self, name, *args, **kw):
        from paper_2512_18134_amd import binding as M
        return getattr(M, name + ("_f16" if self.dt == "f16" else ""))(*args, k_scale=self.scale[0], v_scale=self.scale[1], **kw)

    def bits(self, i):
        return self.pages[i].view(torch.uint8 if self.e4m3 else torch.int16)

    def stored(self, x):
        """What the cache holds for the rows that have a place: bits of the elements, exponent bytes, and the values."""
        x = x[self.there]
        if not self.e4m3:
            return x.view(torch.int16), None, x.double()
        value, e = R.e4m3_row(x)
        q = value / torch.tensor(2.0, dtype=torch.float64) ** e[..., None]
        return q.float().to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8), value

    def check_written(self, before):
        """The pool as it was but for the written places."""
        for i, x in enumerate((self.k, self.v)):
            want, units, _ = self.stored(x)
            got = self.bits(i)[self.page_of.cuda(), :, self.place.cuda()].cpu()
            same = got == want
            if self.e4m3:                                  # either zero
                same |= (got & 0x7f == 0) & (want & 0x7f == 0)
                assert torch.equal(self.scale[i][self.page_of.cuda(), :, self.place.cuda()].cpu(), units)
            assert same.all()
            if before is not None:
                kept = torch.ones(self.bits(i).shape[:1] + self.bits(i).shape[2:3], dtype=torch.bool, device="cuda")
                kept[self.page_of.cuda(), self.place.cuda()] = False
                kept = kept[:, None].expand(-1, self.H, -1)
                assert torch.equal(self.bits(i)[kept], before[0][i][kept])
                if self.e4m3:
                    assert torch.equal(self.scale[i][kept], before[1][i][kept])

    def check_read(self, k, v):
        for x, y in ((self.k, k), (self.v, v)):
            y, (_, _, value) = y.cpu(), self.stored(x)
            assert torch.equal(y[self.there].double(), value.to(R.DT[self.dt]).double())
            assert (y[self.mine & ~self.there] == 0).all()
            assert torch.isnan(y[~self.mine].float()).all(), "rows of nobody were written"


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)])
@pytest.mark.parametrize("D, H, T, page", SIZES)
def test_runs_are_written_where_they_belong_and_read_back(D, H, T, page, dt, e4m3):
    s = Rows(D, H, T, page, dt, e4m3)
    for i in range(2):
        s.bits(i).random_(0, 100)
        if e4m3:
            s.scale[i].random_(100, 130)
    before = [s.bits(i).clone() for i in range(2)], [x if x is None else x.clone() for x in s.scale]
    assert 0 < int((s.mine & ~s.there).sum()) < int(s.there.sum())
    s.call("attn_cache_write", s.k.cuda(), s.v.cuda(), *s.pages, *s.index)
    s.check_written(before)
    # heads first, as the dense forward takes them
    out = [torch.full((H, T, D), float("nan"), dtype=R.DT[dt], device="cuda").transpose(0, 1) for _ in "kv"]
    s.check_read(*s.call("attn_cache_read", *s.pages, *s.index, T, k=out[0], v=out[1]))
    # slices of a projection's rows in, tokens of a wider tensor out
    for i in range(2):
        s.bits(i).copy_(before[0][i])
        if e4m3:
            s.scale[i].copy_(before[1][i])
    rows = torch.cat([s.k[:, :1], s.k, s.v], 1).cuda()
    s.call("attn_cache_write", rows[:, 1:1 + H], rows[:, 1 + H:], *s.pages, *s.index)
    s.check_written(before)
    wide = torch.full((T, 2 * H + 1, D), float("nan"), dtype=R.DT[dt], device="cuda")
    s.check_read(*s.call("attn_cache_read", *s.pages, *s.index, T, k=wide[:, :H], v=wide[:, H:2 * H]))
    assert torch.isnan(wide[:, 2 * H].float()).all()


@pytest.mark.parametrize("dt, e4m3", [("bf16", False), ("f16", True)])
def test_runs_in_pages_far_behind_the_pools_start(dt, e4m3):
    """Pools of more than 2^32 elements, of which the last pages are used."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    D, H, T, page = SIZES[2]
    s = Rows(D, H, T, page, dt, e4m3, n_pages=(2 ** 32 + 2 ** 31) // (H * page * D))
    s.call("attn_cache_write", s.k.cuda(), s.v.cuda(), *s.pages, *s.index)
    s.check_written(None)
    out = [torch.full((T, H, D), float("nan"), dtype=R.DT[dt], device="cuda") for _ in "kv"]
    s.check_read(*s.call("attn_cache_read", *s.pages, *s.index, T, k=out[0], v=out[1]))
