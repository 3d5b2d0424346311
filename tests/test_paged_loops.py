"""The generated loops of the attention over a paged cache (csrc/gen_attn_paged_loop.py): the hazard rules that the hardware does
not enforce, on the emitted text, as for the dense loops; and the scalar program's run: every wave of a workgroup meets the
same barriers, brings every tile once and from the window's entry for that tile, over walks of several windows."""
import os
import re
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "paper_2512_18134_amd", "csrc"))

import asm_emit  # noqa: E402
import gen_attn_paged_loop as gen  # noqa: E402

NAMES = list(gen.CONFIGS)


def emitted(name, dtype="bf16"):
    g = gen.PagedGen(name, dtype)
    g.generate()
    return g, [l.replace("%=", "") for l in g.lines]


def clamped_loads(g, tag):
    if g.LS == 0:
        return ["KSLOW%s_" % tag, "VSLOW%s_" % tag]
    return ["KSLOW%s_" % tag] + ["LD%d_%s_" % (n, tag) for n in range(1, 2 * g.NLD)]


def scalar_written_by_vector(path):
    """Wait states between a v_readlane and the first load through the scalar it wrote (at least five are needed)."""
    t, written = 0, {}
    for ins in path:
        op, dst, src = asm_emit.parse(ins)
        if op == "v_readlane_b32":
            for r in dst:
                written[r] = t
        elif op.startswith("global_load"):
            for r in src:
                if r in written:
                    assert t - written[r] > 5, ins
        elif not op.startswith("s_waitcnt"):
            for r in dst:
                written.pop(r, None)
        t += asm_emit.wait_states(ins)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", NAMES)
def test_main_path_and_detours_obey_the_hazard_rules(name, dtype):
    g, lines = emitted(name, dtype)
    paths = [[]]
    for b in range(4):
        special = "SPECIAL%d_" % b
        paths += [["SLOW%d_" % b], [special] + clamped_loads(g, b), [special, "NOMASK%d_" % b] + clamped_loads(g, b),
                  [special, "FRESH%d_" % b, "WHOLE%d_" % b], [special, "FRESH%d_" % b, "PAGE%d_0_" % b],
                  [special, "TOPL%d_" % b, "DONE_"], [special, "FRESH%d_" % b, "NOMASK%d_" % b, "TOPL%d_" % b, "SLOWL%d_" % b, "DONE_"]]
    paths += [["SPECIALF_"] + clamped_loads(g, "F"), ["SPECIALF_", "FRESHF_", "NOMASKF_"] + clamped_loads(g, "F")]
    for take in paths:
        path = asm_emit.walk(lines, take=take, loop_label="BODY0_", loop_visits=2)
        assert asm_emit.check_stream(path) == len(path), take
        scalar_written_by_vector(path)
    # one tile, and a wave that keeps step, with a window filled meanwhile
    for take in (["SPECIALF_", "FRESHF_"] + clamped_loads(g, "F") + ["SPECIAL1_", "EXIT1_"],
                 ["SPECIAL2_", "FRESH2_", "TOPL2_", "OWED2_", "STANDBYNEXT_"], ["SPECIAL3_", "TOPL3_", "OWED3_", "FRESHSB_"]):
        path = asm_emit.walk(lines, take=take, loop_label="STANDBY_", loop_visits=3)
        assert asm_emit.check_stream(path) == len(path), take
        scalar_written_by_vector(path)


def run(g, lines, n, n_wave, t_full, j_mask, wave=0, missing=0):
    """Loads of one wave's run, by barrier interval; the windows are played back by lane."""
    first = {"tile": 0}          # the windows hold tiles first .. first + 63

    def lanes(what, lane, S):
        if isinstance(what, str):
            if what.startswith("v_mbcnt_lo"):
                first["tile"] = S[g.s_j]
            return None
        if what is None:
            return 0
        tile = first["tile"] + (lane - first["tile"]) % 64
        return tile * g.TB if (what - g.WIN) % 2 == 0 else 0
    kv_last = t_full * g.BN + 4
    sg = {g.s_ntiles: n, g.s_nw: n_wave, g.s_tfull: t_full, g.s_jmask: j_mask, g.s_ldsk: 1 << 20, g.s_ldsv: 1 << 21, g.s_kbase: 0,
          g.s_vbase: 0, g.s_posbase: 8 * wave, g.s_end8: kv_last & ~7, g.s_plog2: 4, g.s_npages: 1, g.s_missing: missing,
          g.s_kvlast: kv_last, g.s_key0: 0}
    ev = asm_emit.run_scalar(lines, sg, g.BN, g.TB, {"k": (-1, g.s_kptr), "v": (-1, g.s_vptr)}, lanes=lanes)
    out = []
    for e in ev:
        if e[0] == "barrier":
            out.append([])
        else:
            out[-1].append(e[1:])
    return out


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6, 9, 55, 56, 57, 60, 64, 113, 200])
def test_every_wave_meets_every_barrier_and_brings_every_tile(name, n):
    g, lines = emitted(name)
    for t_full in (n, n - 1, n + 3):
        for j_mask in sorted({0, n // 2, n}):
            full = run(g, lines, n, n, t_full, j_mask)
            assert len(full) == n
            for j, loads in enumerate(full):
                want = [("k", j + 4, j % 4)] * g.NLD + [("v", j + 2, (j + 2) % 4)] * g.NLD
                if j == n - 1 and n > 1:
                    want = []
                got = sorted((w, t, (a - ((1 << 20) if w == "k" else (1 << 21))) // g.TB) for w, t, a in loads)
                assert got == sorted(want), (n, t_full, j_mask, j)
            for n_wave in sorted({1, 2, n // 2, n - 1} & set(range(1, n))):
                part = run(g, lines, n, n_wave, t_full, j_mask, wave=1)
                assert [sorted(x) for x in part] == [sorted(x) for x in full], (n, n_wave, t_full, j_mask)
    assert run(g, lines, n, n, n, 0, missing=1) == run(g, lines, n, n, n, 0)


def test_the_window_is_filled_before_it_is_left():
    """Between two fillings the pointers ask for tiles up to REFRESH - 1 + 5 behind the filling's first."""
    assert gen.REFRESH + 4 < gen.WINDOW
    for name in NAMES:
        _, lines = emitted(name)
        assert sum(bool(re.match(r"\s*v_readlane", l)) for l in lines) % 4 == 0
