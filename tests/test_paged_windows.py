"""The vector side of the paged loops' rare sections (csrc/gen_attn_paged_loop.py), executed lane by lane from the emitted text: the
addresses that a refilled window holds, and which keys a tile loses to pages that are missing."""
import os
import random
import re
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "paper_2512_18134_amd", "csrc"))

import gen_attn_paged_loop as gen  # noqa: E402

U32 = np.uint64(0xffffffff)
LANES = np.arange(64, dtype=np.uint64)


def section(lines, label):
    """The instructions between the branch to `label` and the label."""
    at = next(i for i, l in enumerate(lines) if re.match(r"s_cbranch\w*\s+%s$" % label, l))
    end = lines.index(label + ":")
    return lines[at + 1:end]


class Wave:
    """Registers of a wave, 32 bits to a lane, and what the sections use of the instructions."""

    def __init__(self, scalars, load):
        self.s, self.v, self.vcc, self.load = dict(scalars), {}, None, load

    def value(self, x):
        if re.fullmatch(r"v\d+", x):
            return self.v[int(x[1:])]
        n = self.s[int(x[1:])] if re.fullmatch(r"s\d+", x) else int(x, 0)
        return np.full(64, n & 0xffffffff, dtype=np.uint64)

    def run(self, lines):
        for l in lines:
            op, rest = (l.split(None, 1) + [""])[:2]
            a = [x.strip() for x in rest.split(",")]
            if op in ("s_waitcnt", "s_nop") or op.startswith("s_add_i32") or op.startswith("s_min_i32"):
                continue                                          # (the scalar program has a test of its own)
            signed = lambda x: x.astype(np.uint32).astype(np.int32)
            if op == "v_cmp_gt_u32":
                assert a[0] == "vcc"
                self.vcc = self.value(a[1]) > self.value(a[2])
                continue
            x = [self.value(y) for y in a[1:] if y != "vcc" and not y.startswith("s[")]
            if op == "v_mbcnt_lo_u32_b32":
                r = np.minimum(LANES, np.uint64(32)) + x[1]
            elif op == "v_mbcnt_hi_u32_b32":
                r = np.maximum(LANES, np.uint64(32)) - np.uint64(32) + x[1]
            elif op == "v_subrev_u32":
                r = x[1] - x[0]
            elif op == "v_add_u32":
                r = x[0] + x[1]
            elif op == "v_and_b32":
                r = x[0] & x[1]
            elif op == "v_lshlrev_b32":
                r = x[1] << (x[0] & np.uint64(31))
            elif op == "v_lshrrev_b32":
                r = x[1] >> (x[0] & np.uint64(31))
            elif op == "v_min_i32":
                r = np.minimum(signed(x[0]), signed(x[1])).astype(np.int64).astype(np.uint64)
            elif op == "v_mov_b32":
                r = x[0]
            elif op == "v_mul_lo_u32":
                r = x[0] * x[1]
            elif op == "v_mul_hi_u32":
                r = x[0] * x[1] >> np.uint64(32)
            elif op == "v_add_co_u32":
                r = x[0] + x[1]
                self.vcc = r > U32
            elif op == "v_addc_co_u32":
                assert a[4] == "vcc"
                r = x[0] + x[1] + self.vcc.astype(np.uint64)
                self.vcc = r > U32
            elif op == "v_cndmask_b32":
                r = np.where(self.vcc, x[1], x[0])
            elif op == "global_load_dword":
                r = self.load(x[0])
            else:
                raise AssertionError("not modelled: " + l)
            self.v[int(a[0][1:])] = r & U32


def emitted(name):
    g = gen.PagedGen(name, "bf16")
    g.generate()
    return g, [l.replace("%=", "") for l in g.lines]


@pytest.mark.parametrize("tag", ["F", "0", "1", "2", "3", "SB"])
@pytest.mark.parametrize("name", list(gen.CONFIGS))
def test_a_refilled_window_holds_the_tiles_from_the_current_one_on(name, tag):
    g, lines = emitted(name)
    text = section(lines, "FRESH%s_" % tag)
    rng = random.Random(5)
    for j, key0, kv, page_log2, H_kv, n_pages in ((56, 0, 4500, 4, 8, 3000), (57, 64, 30000, 8, 1, 1 << 20), (112, 640, 9000, 5, 3, 70000),
                                                  (500, 0, 16011, 6, 16, 2 ** 31 - 1), (13, 1024, 2000, 7, 2, 9), (0, 0, 1, 4, 1, 2)):
        wave = rng.randrange(g.NW)
        page_bytes = (H_kv << page_log2) * g.ROWB
        table = [rng.choice([rng.randrange(n_pages), n_pages - 1, rng.randrange(n_pages), n_pages, -1, 2 ** 31 - 1, -2 ** 31])
                 for _ in range((kv - 1 >> page_log2) + 1)]
        k_head, v_head, zero = (rng.randrange(1 << 47) & ~15 for _ in range(3))
        end8 = kv - 1 & ~7
        words = lambda r, x: {r: x & 0xffffffff, r + 1: x >> 32}
        scalars = {g.s_j: j, g.s_posbase: key0 + 8 * wave, g.s_end8: end8, g.s_plog2: page_log2, g.s_pmask: (1 << page_log2) - 1,
                   g.s_pbytes: page_bytes, g.s_npages: n_pages, **words(g.s_kbase, k_head), **words(g.s_vbase, v_head),
                   **words(g.s_zero, zero)}
        w = Wave(scalars, lambda at: np.array([table[int(x) // 4] & 0xffffffff for x in at], dtype=np.uint64))
        w.run(text)
        for lane in range(64):
            tile = j + (lane - j) % 64
            pos = min(key0 + 8 * wave + g.BN * tile, end8)
            page = table[pos >> page_log2]
            for head, r in ((k_head, g.WIN), (v_head, g.WIN + 2)):
                want = head + page * page_bytes + (pos & (1 << page_log2) - 1) * g.ROWB if 0 <= page < n_pages else zero
                assert int(w.v[r][lane]) | int(w.v[r + 1][lane]) << 32 == want, (lane, tile, page)


@pytest.mark.parametrize("tag", ["F", "0", "1", "2", "3"])
@pytest.mark.parametrize("name", list(gen.CONFIGS))
def test_keys_without_a_page_are_masked_sixteen_at_a_time(name, tag):
    """The scores of a tile whose pages are there or not, in every combination."""
    g, lines = emitted(name)
    text = section(lines, "WHOLE%s_" % tag)
    scores = g.bufs(0 if tag == "F" else int(tag))[0]
    n_pages, page_log2, kv = 50, 4, 10 ** 6
    for present in range(1 << g.BN // 16):
        j, key0 = 37, 192
        S = {g.s_j: j, g.s_key0: key0, g.s_kvlast: kv - 1, g.s_plog2: page_log2, g.s_npages: n_pages}
        masked, i, scc = set(), 0, 0
        first = key0 + j * g.BN >> page_log2
        num = lambda x: S[int(x[1:])] if x[0] == "s" else int(x, 0)
        while i < len(text):
            op, rest = (text[i].split(None, 1) + [""])[:2]
            a = [x.strip() for x in rest.split(",")]
            i += 1
            if op.endswith(":") or op == "s_waitcnt":
                continue
            if op == "s_cbranch_scc1":
                i = text.index(a[0] + ":") if scc else i
            elif op == "s_cmp_lt_u32":
                scc = num(a[0]) & 0xffffffff < num(a[1]) & 0xffffffff
            elif op == "s_load_dword":
                page = num(a[2]) // 4 - first
                assert 0 <= page < g.BN // 16
                S[int(a[0][1:])] = 7 if present >> page & 1 else 0xffffffff
            elif op == "v_mov_b32":
                assert a[1] == "v%d" % g.NEGINF
                masked.add(int(a[0][1:]))
            else:
                S[int(a[0][1:])] = {"s_lshl_b32": lambda x, y: x << y, "s_lshr_b32": lambda x, y: x >> y, "s_add_i32": lambda x, y: x + y,
                                    "s_min_i32": min}[op](num(a[1]), num(a[2]))
        # register r of an accumulator's 16 holds the keys r % 4 + 8 (r / 4) of its 32, and in the other half of the wave 4 behind
        want = set()
        for sb in range(g.BN // 32):
            for r in range(16):
                parts = {(32 * sb + r % 4 + 8 * (r // 4) + 4 * half) // 16 for half in (0, 1)}
                assert len(parts) == 1
                if not present >> parts.pop() & 1:
                    want |= {g.s_reg(scores, qb, sb, 0, r) for qb in range(g.QB)}
        assert masked == want, present
