"""The compiled kernels of trees of drafts and of eviction (hipcc -S): no scratch memory, no spilled vector registers, and as many workgroups on a
compute unit as their launches count on."""
import os
import re
import subprocess

import pytest

from test_compiled_serving_kernels import ROOT, metadata


def listing(source, tmp_path):
    from paper_2512_18134_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not installed")
    out = str(tmp_path / "kernels.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", "-o", out,
                                      os.path.join(ROOT, "paper_2512_18134_amd", "csrc", source + ".hip")],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    return open(out).read()


def registers(text):
    found, name = {}, None
    for key, value in re.findall(r"\n\s+\.(name|vgpr_count):\s+(\S+)", text):
        if key == "name":
            name = value
        else:
            found[name] = int(value)
    return found


@pytest.mark.parametrize("source, kernels", [("attn_tree", 40), ("attn_weigh", 24), ("attn_evict", 10)])
def test_no_scratch_no_spills_and_room_for_the_workgroups(source, kernels, tmp_path):
    text = listing(source, tmp_path)
    found = metadata(text)
    assert len(found) >= kernels
    assert {k: v for k, v in found.items() if v != (0, 0)} == {}
    for name, vgprs in registers(text).items():
        waves = 512 // -(-vgprs // 8 * 8)                  # of a SIMD
        if "attn_paged_tiles_kernel" in name:              # <D, type, e4m3, tree, 32-row blocks>
            three = re.search(r"ILi(64|128)E", name) and "Lb1ELi1EE" in name
            assert waves >= (3 if three else 2), (name, vgprs)
        elif "attn_weigh_tiles_kernel" in name:
            assert waves >= 2, (name, vgprs)               # two workgroups to a compute unit
        elif "attn_select_part_kernel" in name:
            assert waves >= 4, (name, vgprs)               # two of 512 threads
