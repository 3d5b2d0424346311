"""Host side of the serving launches: what a call launches agrees with the kernels that were compiled."""
import os
import re
import subprocess

import pytest

import serving_launches as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def registers(tmp_path):
    """{kernel: vector registers of a lane} of the attention over the paged cache, from the compiler's own listing."""
    from paper_2512_18134_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not installed")
    out = str(tmp_path / "kernels.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", "-o", out,
                                      os.path.join(ROOT, "paper_2512_18134_amd", "csrc", "attn_paged.hip")],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    found, name = {}, None
    for key, value in re.findall(r"\n\s+\.(name|vgpr_count):\s+(\S+)", open(out).read()):
        if key == "name":
            name = value
        else:
            found[name] = int(value)
    return found


def test_a_call_is_cut_for_the_workgroups_that_the_chip_holds(tmp_path):
    """PagedParams::target against what registers and LDS of the launched kernel let 256 compute units hold: 512 registers of a
    SIMD's lane in eights, 160 KB of LDS."""
    have = registers(tmp_path)
    sizes = [(D, rows, e4m3, dt) for D in (64, 128, 256) for rows in (1, 20, 60, 200) for e4m3 in (False, True)
             for dt in ("bf16", "f16")]
    calls = [L.paged(rows, 1, 8, 8, D, 16, 1000, 1000, rows, dt, e4m3) for D, rows, e4m3, dt in sizes]
    seen = set()
    for size, (rc, lines) in zip(sizes, L.launches(tmp_path, calls)):
        assert rc == 0
        main = [x for x in lines if "merge" not in x["kernel"]]
        assert len(main) == 1 and len(lines) == 2
        x = main[0]
        waves = x["threads"] // 64
        per_simd = 512 // -(-have[x["kernel"]] // 8 * 8)
        per_cu = min(per_simd * 4 // waves, 160 * 1024 // x["lds"])
        assert x["target"] == 256 * min(per_cu, 2), (size, L.template(x["kernel"]), have[x["kernel"]])
        seen.add(x["kernel"])
    assert len(seen) == 3 * 4 * 4 - 4               # (D = 256 has no tiles of 64 rows)


def test_the_cache_tests_sizes_are_written_and_read_in_runs(tmp_path):
    """The kernel that takes runs of tokens, in all its variants, is what the sizes of test_cache_runs_gpu.py launch."""
    import test_cache_runs_gpu as C
    calls = [L.rows(what, T, len(C.batch(T, page, 91)[0]), H, D, page, 1 << 20, 64, dt, e4m3)
             for D, H, T, page in C.SIZES for what in ("write", "read") for dt in ("bf16", "f16") for e4m3 in (False, True)]
    seen = set()
    for call, (rc, lines) in zip(calls, L.launches(tmp_path, calls)):
        assert rc == 0 and len(lines) == 1
        assert "attn_cache_run_kernel" in lines[0]["kernel"], call
        seen.add(lines[0]["kernel"])
    assert len(seen) == 3 * 2 * 2 * 2
    for D, H, T, page in C.SIZES:
        news, _, front, behind = C.batch(T, page, 91)
        assert T % 8 and news[-1] > 0 and front + sum(news) + behind == T
        start = front
        crowded = 0                                        # empty sequences that begin inside one run of eight tokens
        at = {}
        for n in news:
            if n == 0:
                at[start // 8] = at.get(start // 8, 0) + 1
            start += n
        crowded = max(at.values())
        assert crowded > 64
    assert any(2 * H % (512 // D) for D, H, _, _ in C.SIZES)


def test_the_rope_tests_sizes_take_the_kernels_of_large_calls(tmp_path):
    """How many heads a wave takes is read from the launch's workgroups of four waves; whether it stores past the caches from the
    kernel's last template argument."""
    import test_rope_large_gpu as P
    calls = [L.rope(*size[:6], interleaved=inter) for size in P.SIZES for inter in (0, 1)]
    found = L.launches(tmp_path, calls)
    for i, (rc, lines) in enumerate(found):
        b, hq, hkv, s, d, sections, per_wave, past = P.SIZES[i // 2]
        assert rc == 0 and len(lines) == 1
        name = lines[0]["kernel"]
        lanes = 1
        while 8 * lanes < sum(sections):
            lanes *= 2
        groups = -(-b * s * lanes // 64)
        assert lines[0]["grid"] == -(-groups * -(-(hq + hkv) // per_wave) // 4), (P.SIZES[i // 2], lines[0])
        assert name.split("attn_rope_kernelI")[1].count("Lb1E") == i % 2 + past, name      # INTERLEAVED, PAST
    assert {size[6] for size in P.SIZES} >= {1, 4, 8, 16} and any(size[7] for size in P.SIZES)
