"""Host side of the tree launches: a call has one attention kernel, and its workspace holds partial results for all workgroups that the chip runs at
once -- with fewer a long sequence of few rows would be walked whole."""
import serving_launches as L

TREE_ARGS = '''    elif name.startswith("attn_paged_tree"):
        entry.argtypes = [p] * 11 + [i, p, i, p, q, i] + [i] * 8 + [f, p]
    else:
'''


def tree(lib, T, B, H_q, H_kv, D, page, width, max_q, dt="bf16", e4m3=False):
    strides = {"int64": [H_q * D, D]}
    need = lib.attn_paged_tree_workspace_bytes(T, B, H_q, H_kv, D)
    return ("attn_paged_tree" + ("_f16" if dt == "f16" else ""),
            L._P[:1] + [strides] + L._P[1:10] + [int(e4m3), L._P[10], 2, L._P[11], need, max_q, T, B, H_q, H_kv, D, 1 << 16, page, width, 0.1, None])


def test_one_kernel_with_room_for_its_workgroups(tmp_path, monkeypatch):
    from paper_2512_18134_amd import binding as lib
    assert L.RUN.count("    else:\n") == 1
    monkeypatch.setattr(L, "RUN", L.RUN.replace("    else:\n", TREE_ARGS))
    sizes = [(D, n, G, B, width, dt, e4m3) for D in (64, 128, 256) for n, G in ((1, 1), (5, 3), (5, 4), (16, 4), (24, 4), (33, 4), (64, 8))
             for B, width in ((1, 32), (1, 64), (1, 8192), (40, 8192)) for dt in ("bf16", "f16") for e4m3 in (False, True)]
    calls = [tree(lib, n * B, B, 2 * G, 2, D, 16, width, n, dt, e4m3) for D, n, G, B, width, dt, e4m3 in sizes]
    seen = set()
    for (D, n, G, B, width, dt, e4m3), (rc, lines) in zip(sizes, L.launches(tmp_path, calls)):
        assert rc == 0
        main = [x for x in lines if "merge" not in x["kernel"]]
        assert len(main) == 1 and len(lines) <= 2 and all(x["allowed"] for x in lines)
        x = main[0]
        name = L.template(x["kernel"])
        if x["rounds"]:                                    # (0: whole sequences by eight waves)
            assert x["slots"] >= x["target"] + 64, (D, n, G, B, width, name)
            assert len(lines) == 2 or width * 16 <= 256    # the merge
        if name[0] == "attn_paged_tiles_kernel":
            assert n * G > (64 if D < 256 else 32 if e4m3 else 16)
            assert x["target"] == 256 * (3 if D < 256 and n * G <= 128 else 2)
        seen.add(x["kernel"])
    # by 16 rows (four and eight waves), 32 and 64, and tiles of 128 and 256 rows; D = 256: no eight waves, 32 rows in e4m3 alone, tiles of 128
    assert len(seen) == 2 * (2 * 2 * 6 + (2 + 3))
