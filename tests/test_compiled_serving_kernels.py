"""The compiled kernels of the serving operators (hipcc -S) keep to registers.

Registers in scratch memory cost a wait for every load in flight at each reload; and a register tuple of which the compiler had
put some parts into scratch and others into accumulation registers was once reloaded in part only, which gave wrong results.
So no kernel of these sources may use scratch memory, or spill vector registers anywhere."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def metadata(text):
    """{kernel: (bytes of scratch, vector registers spilled)} from the metadata behind the code."""
    out, scratch, name = {}, None, None
    for line in text.split("\n"):
        m = re.match(r"\s+\.(name|private_segment_fixed_size|vgpr_spill_count):\s+(\S+)$", line)
        if not m:
            continue
        key, value = m.groups()
        if key == "name" and value.startswith("_Z"):
            name = value
        elif key == "private_segment_fixed_size":
            scratch = int(value)
        elif key == "vgpr_spill_count":
            out[name] = (scratch, int(value))
    return out


def test_metadata_is_read():
    text = ("    .name:           _Zone\n    .private_segment_fixed_size: 0\n    .vgpr_spill_count: 0\n"
            "      - .name:           argument\n"
            "    .name:           _Ztwo\n    .private_segment_fixed_size: 12\n    .vgpr_spill_count: 3\n")
    assert metadata(text) == {"_Zone": (0, 0), "_Ztwo": (12, 3)}


@pytest.mark.parametrize("source, kernels", [("attn_rope", 4), ("attn_cache", 20), ("attn_paged", 20)])
def test_no_scratch_and_no_spills(source, kernels, tmp_path):
    from paper_2512_18134_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not installed")
    out = str(tmp_path / "kernels.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", "-o", out,
                                      os.path.join(ROOT, "paper_2512_18134_amd", "csrc", source + ".hip")],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    found = metadata(open(out).read())
    assert len(found) >= kernels
    assert {k: v for k, v in found.items() if v != (0, 0)} == {}
