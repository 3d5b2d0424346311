"""How a call over the paged cache is cut into units (csrc/attn_paged_plan.h), on the host: the device code runs as 64
coroutines (wave_host).  Every row tile and every key of every sequence belongs to exactly one unit, the units fit the launch and
the workspace, and whatever the arrays of lengths hold, nothing points outside."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2512_18134_amd", "csrc")
FIELDS = ("b", "h", "tile", "range", "n_ranges", "n_tiles", "row0", "n_rows", "n", "kv", "key0", "key1", "slot0", "slot")
ALL = 0x7fffffff


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.run(["/opt/rocm/bin/amdclang++", "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-shared",
                    "-I" + os.path.join(HERE, "wave_host"), "-I" + CSRC, "-o", so,
                    os.path.join(HERE, "wave_host", "paged_plan.cpp")], check=True)
    return ctypes.CDLL(so)


def ints(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def plan(lib, start, kv_len, T, H_kv, G, BM, width, page_log2=4, above=0, upto=ALL, target=64, min_range=2, n_slots=None, causal=1, rounds=1, before=None):
    B = len(kv_len)
    n_slots = 4 * target + 64 if n_slots is None else n_slots
    n_wg = (T * G // BM + min(B, T)) * H_kv + target * rounds * (2 if causal else 1) + 64    # the launch's own bound
    start, kv_len = ints(start), ints(kv_len)
    table = np.zeros((B, width), np.int32)
    units = np.zeros((n_wg, 14), np.int32)
    notes = np.full((T + 2, 4), -77, np.int32)                    # a guard row on either side
    before = B > 128 if before is None else before               # the cut is left in a table first, as for so many sequences
    cut = np.full((B + 3, 2), -77, np.int32)
    n = lib.plan_batch(ptr(table), ptr(start), ptr(kv_len), T, B, H_kv, 1, page_log2, width, G, BM, above, upto, target,
                       min_range, n_slots, causal, rounds, n_wg, ptr(units), ctypes.c_void_p(notes.ctypes.data + 16),
                       ctypes.c_void_p(cut.ctypes.data + 8) if before else None)
    assert (cut[0] == -77).all() and (cut[-1] == -77).all()
    assert n >= 0
    assert (notes[0] == -77).all() and (notes[-1] == -77).all()
    return [dict(zip(FIELDS, map(int, u))) for u in units[:n]], notes[1:-1], n_wg, n_slots


CASES = [
    dict(news=[1], kvs=[1], H=1, G=1, BM=16),
    dict(news=[1], kvs=[1000], H=16, G=1, BM=16),
    dict(news=[1] * 64, kvs=[17 * i + 1 for i in range(64)], H=2, G=4, BM=16),
    dict(news=[1] * 65, kvs=[13 * i + 1 for i in range(65)], H=2, G=3, BM=16),
    dict(news=[0, 5, 0, 7, 1, 0], kvs=[0, 900, 30, 7, 5000, 0], H=3, G=5, BM=32),
    dict(news=[40, 1, 300], kvs=[40, 20000, 2300], H=2, G=3, BM=64),
    dict(news=[3, 2], kvs=[0, 1], H=2, G=1, BM=16),                    # rows below position 0
    dict(news=[1] * 200, kvs=[131072] + [40] * 199, H=1, G=8, BM=16),  # one long sequence among short ones
    dict(news=[700], kvs=[131072], H=1, G=4, BM=256),
    dict(news=[0, 0], kvs=[5, 6], H=4, G=2, BM=16),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "B%d_H%d_G%d_BM%d" % (len(c["news"]), c["H"], c["G"], c["BM"]))
@pytest.mark.parametrize("front, behind, rounds, causal", [(0, 0, 1, 1), (3, 4, 4, 0), (1, 0, 3, 1)])
def test_units_cover_every_row_and_key_once(lib, case, front, behind, rounds, causal):
    news, kvs, H, G, BM = (case[k] for k in ("news", "kvs", "H", "G", "BM"))
    start = front + np.concatenate([[0], np.cumsum(news)])
    T = max(1, int(start[-1]) + behind)
    width = max(1, -(-max(kvs) // 16))
    units, notes, n_wg, n_slots = plan(lib, start, kvs, T, H, G, BM, width, rounds=rounds, causal=causal)
    seen, slots = {}, set()
    for u in units:
        b = u["b"]
        assert u["n"] == news[b] and u["kv"] == kvs[b] and u["row0"] == start[b] and u["n_rows"] == news[b] * G
        assert u["n_tiles"] == -(-news[b] * G // BM) and 0 <= u["tile"] < u["n_tiles"] and 0 <= u["h"] < H
        key = (b, u["h"], u["tile"])
        assert (u["key0"], u["key1"]) not in seen.get(key, [])
        seen.setdefault(key, []).append((u["key0"], u["key1"]))
        if u["n_ranges"] > 1:
            assert 0 <= u["slot"] < n_slots and u["slot"] not in slots
            assert u["slot"] == u["slot0"] + (u["range"] * H + u["h"]) * u["n_tiles"] + u["tile"]     # where the merge looks
            slots.add(u["slot"])
    want = {(b, h, t) for b in range(len(news)) for h in range(H) for t in range(-(-news[b] * G // BM))}
    assert set(seen) == want
    for (b, _, _), ranges in seen.items():
        ranges.sort()
        assert ranges[0][0] == 0 and ranges[-1][1] == kvs[b]
        assert all(x[1] == y[0] for x, y in zip(ranges, ranges[1:]))
        assert all(x[0] % 64 == 0 for x in ranges)
    # notes: exactly the tokens of the batch, with their sequence's slots
    of = {u["b"]: u for u in units}
    for t in range(T):
        b = int(np.searchsorted(start, t, side="right")) - 1
        if t < start[0] or t >= start[-1]:
            assert (notes[t] == -77).all()
        else:
            u = of[b]
            assert list(notes[t]) == [u["slot0"], u["n_tiles"], u["n_ranges"], (t - start[b]) * G * 2]


def test_two_kernels_share_a_batch(lib):
    news, kvs = [1, 40, 2, 500], [3000, 3040, 70, 500]
    start = np.concatenate([[0], np.cumsum(news)])
    rows, _, _, _ = plan(lib, start, kvs, int(start[-1]), 2, 4, 64, 200, above=0, upto=64)
    tiles, _, _, _ = plan(lib, start, kvs, int(start[-1]), 2, 4, 128, 200, above=64)
    assert {u["b"] for u in rows} == {0, 2} and {u["b"] for u in tiles} == {1, 3}


def test_a_long_sequence_is_shared_out(lib):
    units, _, _, _ = plan(lib, list(range(9)), [131072] + [64] * 7, 8, 8, 4, 16, 8192, target=128)
    longest = max(u["key1"] - u["key0"] for u in units)
    assert longest <= 131072 * 8 // 128 + 128        # its share of 128 workgroups, to a block


def test_units_fill_the_last_round(lib):
    """Six row tiles of eight heads on 32 workgroups: one range each would be 48 units in two rounds, the second half empty."""
    for rounds, most in ((1, 2.0), (4, 1.51)):
        units, _, _, _ = plan(lib, [0, 24], [64 * 600], 24, 8, 4, 16, 2400, target=32, rounds=rounds, causal=0)
        work = sum(u["key1"] - u["key0"] for u in units)
        longest = max(u["key1"] - u["key0"] for u in units)
        assert -(-len(units) // 32) * longest <= most * work / 32


@pytest.mark.parametrize("H", [1, 2, 3, 4, 5, 8, 12, 16, 20])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 16])
def test_heads_share_xcds_evenly(lib, H, n):
    got = [[ctypes.c_int(), ctypes.c_int()] for _ in range(H * n)]
    for w, (h, t) in enumerate(got):
        lib.layer_place(w, H, n, ctypes.byref(h), ctypes.byref(t))
    got = [(h.value, t.value) for h, t in got]
    assert sorted(got) == [(h, t) for h in range(H) for t in range(n)]
    if H % 8 == 0:
        assert all(len({h for w, (h, _) in enumerate(got) if w % 8 == x}) == H // 8 for x in range(8))


@pytest.mark.parametrize("causal", [0, 1])
def test_few_slots_make_longer_ranges(lib, causal):
    units, _, _, n_slots = plan(lib, [0, 900, 900, 901], [5000, 77, 800], 901, 2, 4, 64, 400, n_slots=230, rounds=4,
                                target=128, causal=causal)
    assert len({u["slot"] for u in units if u["n_ranges"] > 1}) == sum(u["n_ranges"] > 1 for u in units)
    assert all(u["n_ranges"] == 1 or u["slot"] < 230 for u in units) and {u["b"] for u in units} == {0, 2}
    units, _, _, _ = plan(lib, [0, 900, 900, 901], [5000, 77, 800], 901, 2, 4, 64, 400, n_slots=0, causal=causal)
    assert all(u["n_ranges"] == 1 for u in units)


@pytest.mark.parametrize("seed", range(12))
def test_arrays_that_make_no_sense_stay_in_bounds(lib, seed):
    rng = random.Random(seed)
    B, T, H, G, BM = rng.choice([1, 5, 70, 130]), rng.choice([1, 9, 300]), 2, 3, rng.choice([16, 64, 256])
    wild = lambda lo, hi: rng.choice([rng.randint(lo, hi), rng.randint(-2 ** 31, 2 ** 31 - 1), 2 ** 31 - 1, -2 ** 31, 0])
    start = [wild(0, T) for _ in range(B + 1)]
    kvs = [wild(0, 5000) for _ in range(B)]
    units, _, _, n_slots = plan(lib, start, kvs, T, H, G, BM, 64, target=64)
    for u in units:
        assert 0 <= u["b"] < B and 0 <= u["h"] < H and 0 <= u["tile"] < u["n_tiles"] and u["n"] > 0
        assert 0 <= u["row0"] and u["row0"] + u["n"] <= T and u["n_rows"] == u["n"] * G
        assert 0 <= u["key0"] <= u["key1"] <= u["kv"] <= 64 * 16
        assert u["n_ranges"] == 1 or 0 <= u["slot"] < n_slots


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 200, 5000])
def test_sequence_of_a_row(lib, B):
    rng = random.Random(B)
    news = [rng.choice([0, 0, 1, 1, 2, 9]) for _ in range(B)]
    start = ints(2 + np.concatenate([[0], np.cumsum(news)]))
    T = int(start[-1]) + 3
    for t in [0, 1, 2, T - 4, T - 3, T - 1] + [rng.randrange(T) for _ in range(60)]:
        got = lib.sequence_of(ptr(start), T, B, t)
        inside = start[0] <= t < start[-1]
        assert got == (int(np.searchsorted(start, t, side="right")) - 1 if inside else -1), t
    wild = ints([rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in range(B + 1)])
    for t in range(0, T, max(1, T // 20)):
        assert -1 <= lib.sequence_of(ptr(wild), T, B, t) < B


@pytest.mark.parametrize("page_log2", [4, 6, 8])
def test_pages_outside_the_pool_are_no_pages(lib, page_log2):
    table = ints([[0, 6, 7, -1, 2 ** 31 - 1, -2 ** 31, 3]])
    length = ctypes.c_int()
    for kv, most in ((5, 5), (-3, 0), (2 ** 31 - 1, 7 << page_log2), (7 << page_log2, 7 << page_log2)):
        kv_len = ints([kv])
        for i, want in enumerate([0, 6, -1, -1, -1, -1, 3]):
            for pos in (i << page_log2, (i + 1 << page_log2) - 1):
                got = lib.page_of(ptr(table), ptr(kv_len), 0, 7, page_log2, 7, pos, ctypes.byref(length))
                assert length.value == most
                assert got == (want if pos < most else -2)


def test_divisions_without_a_division(lib):
    rng = random.Random(1)
    for G in list(range(1, 70)) + [96, 100, 127, 128, 129, 1000, 65537, 2 ** 20 + 7, 2 ** 29 + 1]:
        for k in [0, 1, 5, 1000, (2 ** 31 - 1) // G] + [rng.randrange(2 ** 31 // G) for _ in range(5)]:
            for row in (k * G - 1, k * G, k * G + 1):
                if 0 <= row < 2 ** 31:
                    assert lib.row_over(row, G) == row // G, (row, G)
    for _ in range(3000):
        b = rng.choice([1, 2, 3, 7, 8, rng.randrange(1, 5000), rng.randrange(1, 2 ** 22)])
        a = rng.choice([0, b - 1, b, b * rng.randrange(1, 50), rng.randrange(2 ** 22), 2 ** 22 - 1, 2 ** 22, 2 ** 31 - 1])
        assert lib.over(a, b) == a // b, (a, b)


@pytest.mark.parametrize("B", [1, 2, 64, 65, 130])
@pytest.mark.parametrize("rounds", [0, 1, 4])
def test_the_table_of_units_says_what_the_workgroups_find(lib, B, rounds):
    """The cut worked out by every workgroup, and once before them: the same units, whatever the lengths (0 among them)."""
    rng = random.Random(B)
    news = [rng.choice([0, 1, 1, 3]) for _ in range(B)]
    news[0] = 2
    kvs = [n + rng.choice([0, 0, 5, 70, 900]) for n in news]
    start = np.concatenate([[0], np.cumsum(news)])
    args = (lib, start, kvs, int(start[-1]), 2, 3, 16, 64)
    one, other = (plan(*args, target=16, rounds=rounds, before=b) for b in (False, True))
    assert one[0] == other[0] and (one[1] == other[1]).all()


@pytest.mark.parametrize("seed", range(4))
def test_a_table_of_arrays_that_make_no_sense_stays_in_bounds(lib, seed):
    rng = random.Random(100 + seed)
    B, T, width = rng.choice([3, 129, 200]), 50, 4
    wild = lambda: rng.choice([-2 ** 31, -1, 0, 7, 30, 50, 51, 2 ** 31 - 1])
    units, _, n_wg, n_slots = plan(lib, [wild() for _ in range(B + 1)], [wild() for _ in range(B)], T, 2, 2, 16, width, before=True)
    assert len(units) <= n_wg
    for u in units:
        assert 0 <= u["b"] < B and 0 <= u["h"] < 2 and 0 <= u["row0"] <= T and u["row0"] + u["n"] <= T
        assert 0 <= u["key0"] <= u["key1"] <= width * 16 and 0 <= u["tile"] < u["n_tiles"]
        assert u["n_ranges"] == 1 or 0 <= u["slot"] < n_slots
