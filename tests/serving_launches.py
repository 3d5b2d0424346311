"""What a serving call launches, on the host: the product library in a process of its own with the stand-in HIP runtime of fake_hip
in front of it, which writes down every launch and, of the attention kernels, how their work is to be cut."""
import json
import os
import subprocess
import sys

import fake_hip

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FIELDS = ("target", "rounds", "most_units", "slots", "rows_above", "rows_upto")

OFFSETS = r"""
#include <stdio.h>
#include "attn_paged_plan.h"
int main() { printf("%s", %s); }
"""

RUN = r"""
import ctypes, json, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
fake.fake_log(sys.argv[3].encode())
lib = ctypes.CDLL(sys.argv[2])
p, i, q, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float
out = []
for name, args in json.load(sys.stdin):
    entry = getattr(lib, name)
    if name.startswith("attn_rope"):
        entry.argtypes = [p] * 8 + [i] * 8 + [p]
    elif name.startswith("attn_cache"):
        entry.argtypes = [p] * 10 + [i] * 8 + [p]
    else:
        entry.argtypes = [p] * 11 + [i, p, q, i] + [i] * 9 + [f, p]
    array = lambda a: (q * len(a["int64"]))(*a["int64"]) if "int64" in a else (i * len(a["int32"]))(*a["int32"])
    rc = entry(*[array(a) if isinstance(a, dict) else a for a in args])
    fake.fake_flush()
    out.append((rc, sum(1 for _ in open(sys.argv[3]))))
print(json.dumps(out))
"""


def _source(offsets):
    """The stand-in, for a library of more kernels, with the plan's fields of attention launches written down."""
    text = fake_hip.SOURCE
    for old, new in (("kernels[256]", "kernels[1024]"), ("n_kernels < 256", "n_kernels < 1024")):
        assert text.count(old) == 1
        text = text.replace(old, new)
    old = '    fprintf(out, "}\\n");\n    return ok ? 0 : 1;\n}\n'
    assert text.count(old) == 1
    dump = '    fprintf(out, ", \\"lds\\": %u", (unsigned)lds);\n    if (strstr(kernels[k].name, "attn_paged"))\n        fprintf(out, "'
    dump += ", ".join([""] + ['\\"%s\\": %%d' % n for n in FIELDS]) + '"'
    dump += "".join(', *(const int *)((const char *)args[0] + %d)' % o for o in offsets) + ');\n'
    return text.replace(old, dump + old)


def launches(tmp_path, calls):
    """(status, [launch]) of each of `calls` -- (entry point, arguments); arrays as {"int64": [...]} or {"int32": [...]}."""
    src, exe = str(tmp_path / "offsets.cpp"), str(tmp_path / "offsets")
    with open(src, "w") as f:
        f.write("#include <stddef.h>\n" + OFFSETS % (" ".join(["%zu"] * len(FIELDS)), ", ".join("offsetof(attn::PagedParams, %s)" % n for n in FIELDS)))
    subprocess.run(["/opt/rocm/bin/amdclang++", "-std=c++17", "-w", "-I" + os.path.join(HERE, "wave_host"),
                    "-I" + os.path.join(ROOT, "paper_2512_18134_amd", "csrc"), "-o", exe, src], check=True)
    offsets = [int(x) for x in subprocess.run([exe], check=True, stdout=subprocess.PIPE).stdout.split()]
    c, so, log = (str(tmp_path / n) for n in ("fake_hip.c", "fake_hip.so", "log"))
    with open(c, "w") as f:
        f.write(_source(offsets))
    subprocess.run([os.environ.get("CC", "gcc"), "-O1", "-shared", "-fPIC", "-w", "-o", so, c], check=True)
    library = os.path.join(ROOT, "paper_2512_18134_amd", "libmi355attn.so")
    done = subprocess.run([sys.executable, "-c", RUN, so, library, log], input=json.dumps(calls), text=True, check=True,
                          stdout=subprocess.PIPE)
    lines, out, at = [json.loads(x) for x in open(log)], [], 0
    for rc, n in json.loads(done.stdout.splitlines()[-1]):
        out.append((rc, lines[at:n]))
        at = n
    return out


# the entry points with sizes only: addresses are numbers that nothing follows
_P = [4096 * (n + 1) for n in range(12)]


def rope(B, H_q, H_kv, S, D, sections, dt="bf16", interleaved=0, inverse=0):
    strides = {"int64": [H_q * S * D, S * D, D] * 2 + [H_kv * S * D, S * D, D] * 2}
    return ("attn_rope" + ("_f16" if dt == "f16" else ""),
            _P[:4] + [strides] + _P[4:6] + [{"int32": list(sections)}, len(sections), B, H_q, H_kv, S, D, interleaved, inverse, None])


def rows(what, T, B, H_kv, D, page, n_pages, width, dt="bf16", e4m3=False):
    strides = {"int64": [H_kv * D, D] * 2}
    return ("attn_cache_" + what + ("_f16" if dt == "f16" else ""),
            _P[:2] + [strides] + _P[2:9] + [int(e4m3), T, B, H_kv, D, n_pages, page, width, None])


def paged(T, B, H_q, H_kv, D, page, n_pages, width, max_q, dt="bf16", e4m3=False, causal=1):
    strides = {"int64": [H_q * D, D]}
    return ("attn_paged_fwd" + ("_f16" if dt == "f16" else ""),
            _P[:1] + [strides] + _P[1:10] + [int(e4m3), _P[10], 1 << 40, max_q, T, B, H_q, H_kv, D, n_pages, page, width, causal, 0.1, None])


def template(kernel):
    """Name and template arguments of a kernel, as [name, argument, ...] of the demangled text."""
    text = subprocess.run(["c++filt", kernel], check=True, stdout=subprocess.PIPE, text=True).stdout
    name = text.split("attn::", 1)[1].split("(")[0]
    name, _, args = name.partition("<")
    return [name] + [a.strip().replace("attn::", "") for a in args.rstrip("> ").split(",")]
