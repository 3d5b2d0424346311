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
