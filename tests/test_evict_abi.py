"""What attn_cache_weigh, attn_cache_select and attn_cache_move refuse, on the host, before any HIP call (no GPU needed)."""
import pytest
import torch

from test_serving_abi import OK, arr, b, caller  # noqa: F401

FAR = 1 << 40
WEIGH = [("q", OK), ("strides", arr([512, 64])), ("lse", OK), ("k_pages", OK), ("k_scale", OK), ("table", OK), ("start", OK), ("kv_len", OK),
         ("kind", 1), ("weights", OK), ("out", OK), ("stamps", OK), ("seen", OK), ("decay", 1.0), ("max_q", 1), ("T", 3), ("B", 2),
         ("H_q", 4), ("H_kv", 2), ("D", 64), ("n_pages", 9), ("page_size", 16), ("width", 4), ("causal", 1), ("scale", 0.125), ("stream", 0)]
SELECT = [("weights", OK), ("stamps", OK), ("seen", OK), ("kv_len", OK), ("keep", OK), ("dst", OK), ("src", OK), ("new_len", FAR),
          ("sinks", 0), ("recent", 0), ("ws", OK), ("ws_bytes", 1 << 50), ("B", 2), ("H_kv", 2), ("width", 64), ("moves", 8), ("stream", 0)]
MOVE = [("k_pages", OK), ("v_pages", OK), ("k_scale", OK), ("v_scale", OK), ("table", OK), ("dst", OK), ("src", OK), ("kind", 1),
        ("weights", OK), ("stamps", OK), ("heads", 2), ("moves", 8), ("B", 2), ("H_kv", 2), ("D", 64), ("n_pages", 9), ("page_size", 16),
        ("width", 4), ("stream", 0)]


@pytest.mark.parametrize("suffix", ["", "_f16"])
def test_weigh_refusals(b, suffix):  # noqa: F811
    f = caller(b, "attn_cache_weigh" + suffix, WEIGH)
    for n in ("q", "strides", "lse", "k_pages", "k_scale", "table", "start", "kv_len", "out", "stamps", "seen"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    assert f(weights=None, start=OK + 2) == b.ATTN_ERR_ALIGN and f(stamps=None, seen=None, start=OK + 2) == b.ATTN_ERR_ALIGN
    for n in ("T", "B", "H_q", "H_kv", "n_pages", "width", "max_q"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    assert f(H_q=5) == b.ATTN_ERR_SHAPE and f(T=1 << 30) == b.ATTN_ERR_SHAPE and f(width=1 << 27) == b.ATTN_ERR_SHAPE
    assert f(B=1 << 30, width=1 << 26) == b.ATTN_ERR_SHAPE and f(B=(1 << 30) + 1, start=OK + 2) == b.ATTN_ERR_SHAPE
    for D in (0, 32, 96, 512):
        assert f(D=D) == b.ATTN_ERR_UNSUPPORTED_D
    for size in (0, 8, 24, 512):
        assert f(page_size=size) == b.ATTN_ERR_UNSUPPORTED
    assert f(kind=3) == b.ATTN_ERR_UNSUPPORTED
    for i in range(2):
        for bad in (-8, 4, 1 << 41):
            s = [512, 64]
            s[i] = bad
            assert f(strides=arr(s)) == b.ATTN_ERR_SHAPE
    size = 2 * 2 * 64 * 4
    for off in (16, size - 16, 16 - size):
        assert f(weights=FAR + off, out=FAR) == b.ATTN_ERR_SHAPE
    for off in (0, size, -size):
        assert f(weights=FAR + off, out=FAR, start=OK + 2) == b.ATTN_ERR_ALIGN
    for n in ("q", "k_pages", "k_scale", "stamps"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    assert f(weights=OK + 8, out=OK + 8) == b.ATTN_ERR_ALIGN
    for n in ("lse", "table", "start", "kv_len", "seen"):
        assert f(**{n: OK + 2}) == b.ATTN_ERR_ALIGN
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert f(scale=s) == b.ATTN_ERR_SCALE
    for d in (-1.0, float("nan"), float("inf")):
        assert f(decay=d) == b.ATTN_ERR_SCALE


def test_select_refusals(b):  # noqa: F811
    f = caller(b, "attn_cache_select", SELECT)
    for n in ("weights", "stamps", "seen", "kv_len", "keep", "dst", "src", "new_len"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    assert f(stamps=None, seen=None, dst=OK + 2) == b.ATTN_ERR_ALIGN
    for n in ("B", "H_kv", "width", "moves"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -16}) == b.ATTN_ERR_SHAPE
    assert f(sinks=-1) == b.ATTN_ERR_SHAPE and f(recent=-1) == b.ATTN_ERR_SHAPE
    assert f(width=72) == b.ATTN_ERR_SHAPE and f(width=(1 << 30) + 16) == b.ATTN_ERR_SHAPE
    assert f(B=1 << 21) == b.ATTN_ERR_SHAPE and f(B=1 << 20, width=1 << 20) == b.ATTN_ERR_SHAPE
    assert f(B=1 << 20, moves=1 << 20) == b.ATTN_ERR_SHAPE
    for n in ("kv_len", "keep", "seen"):
        for off in (-4, 0, 4):
            assert f(**{n: FAR + off}) == b.ATTN_ERR_SHAPE
    for n in ("weights", "stamps"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    for n in ("seen", "kv_len", "keep", "dst", "src"):
        assert f(**{n: OK + 2}) == b.ATTN_ERR_ALIGN
    assert f(new_len=FAR + 2) == b.ATTN_ERR_ALIGN
    need = b.attn_cache_select_workspace_bytes
    assert need(2, 2, 16384) == 0 and f(ws=None, ws_bytes=0, dst=OK + 2) == b.ATTN_ERR_ALIGN
    assert need(2, 2, 16400) > 0 and need(2, 2, 16400) % 16 == 0
    assert f(width=16400, ws=None) == b.ATTN_ERR_NULL and f(width=16400, ws=OK + 8) == b.ATTN_ERR_ALIGN
    assert f(width=16400, ws_bytes=need(2, 2, 16400) - 1) == b.ATTN_ERR_WORKSPACE
    for bad in ((0, 2, 64), (2, 0, 64), (2, 2, 0), (2, 2, 24), (2, 2, (1 << 30) + 16), (1 << 21, 2, 64)):
        assert need(*bad) == -1
    assert f(B=1 << 20, width=1 << 17) == b.ATTN_ERR_SHAPE                        # 2^24 workgroups of 512 threads


def test_move_refusals(b):  # noqa: F811
    f = caller(b, "attn_cache_move", MOVE)
    for n in ("k_pages", "v_pages", "k_scale", "v_scale", "table", "dst", "src"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    assert f(kind=0, k_scale=None, v_scale=None, weights=None, stamps=None, dst=OK + 2) == b.ATTN_ERR_ALIGN
    for n in ("B", "H_kv", "n_pages", "width", "moves", "heads"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    assert f(heads=3) == b.ATTN_ERR_SHAPE and f(heads=1, dst=OK + 2) == b.ATTN_ERR_ALIGN
    for D in (0, 32, 96, 512):
        assert f(D=D) == b.ATTN_ERR_UNSUPPORTED_D
    for size in (0, 8, 24, 512):
        assert f(page_size=size) == b.ATTN_ERR_UNSUPPORTED
    assert f(kind=2) == b.ATTN_ERR_UNSUPPORTED
    assert f(width=1 << 27) == b.ATTN_ERR_SHAPE and f(n_pages=2 ** 31 - 1, H_kv=1 << 10, heads=1) == b.ATTN_ERR_SHAPE
    assert f(B=(1 << 30) + 1) == b.ATTN_ERR_SHAPE and f(B=1 << 30, moves=1 << 20) == b.ATTN_ERR_SHAPE
    assert f(B=1 << 23) == b.ATTN_ERR_SHAPE                # 2^24 workgroups of 256 threads
    for n in ("k_pages", "v_pages", "k_scale", "v_scale"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    for n in ("table", "dst", "src", "weights", "stamps"):
        assert f(**{n: OK + 2}) == b.ATTN_ERR_ALIGN


def test_the_binding_refuses_what_is_not_on_the_gpu_or_does_not_fit(b):  # noqa: F811
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError):
        b.attn_cache_weigh(bf(3, 2, 64), torch.zeros(3, 2), bf(4, 2, 16, 64), i32(1, 4), i32(2), i32(1), torch.zeros(1, 2, 64))
    with pytest.raises(TypeError):
        b.attn_cache_select(torch.zeros(1, 2, 64), i32(1), i32(1), 8)
    with pytest.raises(TypeError):
        b.attn_cache_move(bf(4, 2, 16, 64), bf(4, 2, 16, 64), i32(1, 4), i32(1, 2, 8), i32(1, 2, 8))
    with pytest.raises(TypeError):
        b.attn_cache_move(bf(4, 2, 16, 64).float(), bf(4, 2, 16, 64), i32(1, 4), i32(1, 2, 8), i32(1, 2, 8))
