"""What the serving entry points refuse, on the host, before any HIP call (no GPU needed)."""
import ctypes

import pytest
import torch

OK = 0x1000      # aligned, never dereferenced on a validation error


@pytest.fixture(scope="module")
def b():
    from paper_2512_18134_amd import binding
    return binding


def arr(values, kind=ctypes.c_longlong):
    return (kind * len(values))(*values)


def caller(b, entry, spec):
    def call(**kw):
        assert set(kw) <= {n for n, _ in spec}
        return getattr(b._lib, entry)(*[kw.get(n, d) for n, d in spec])
    return call


ROPE = [("q", OK), ("q_out", OK), ("k", OK), ("k_out", OK), ("strides", arr([1 << 20, 1 << 10, 64] * 4)), ("pos", OK),
        ("freq", OK), ("sections", arr([8, 24], ctypes.c_int)), ("n_axes", 2), ("B", 1), ("H_q", 4), ("H_kv", 2), ("S", 5),
        ("D", 64), ("interleaved", 0), ("inverse", 0), ("stream", 0)]
ROWS = [("k", OK), ("v", OK), ("strides", arr([512, 64] * 2)), ("k_pages", OK), ("v_pages", OK), ("k_scale", OK), ("v_scale", OK),
        ("table", OK), ("start", OK), ("kv_len", OK), ("kind", 1), ("T", 3), ("B", 2), ("H_kv", 2), ("D", 64), ("n_pages", 9),
        ("page_size", 16), ("width", 4), ("stream", 0)]
PAGED = [("q", OK), ("strides", arr([512, 64])), ("o", OK), ("lse", OK), ("k_pages", OK), ("v_pages", OK), ("k_scale", OK),
         ("v_scale", OK), ("table", OK), ("start", OK), ("kv_len", OK), ("kind", 1), ("ws", OK), ("ws_bytes", 1 << 40), ("max_q", 1),
         ("T", 3), ("B", 2), ("H_q", 4), ("H_kv", 2), ("D", 64), ("n_pages", 9), ("page_size", 16), ("width", 4), ("causal", 1),
         ("scale", 0.125), ("stream", 0)]


@pytest.mark.parametrize("suffix", ["", "_f16"])
def test_rope_refusals(b, suffix):
    f = caller(b, "attn_rope" + suffix, ROPE)
    for n in ("q", "q_out", "k", "k_out", "strides", "pos", "freq", "sections"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    assert f(H_kv=0, k=None, k_out=None, q=OK + 8) == b.ATTN_ERR_ALIGN        # q alone needs no k
    for n in ("B", "H_q", "S", "n_axes"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    assert f(H_kv=-1) == b.ATTN_ERR_SHAPE and f(n_axes=5) == b.ATTN_ERR_SHAPE
    for D in (0, 32, 96, 512):
        assert f(D=D) == b.ATTN_ERR_UNSUPPORTED_D
    for s in ([0, 0], [4, 0], [8, 4], [32, 8], [-8, 16], [2 ** 31 - 1, 9]):
        assert f(sections=arr(s, ctypes.c_int)) == b.ATTN_ERR_SHAPE
    for i in range(12):
        for bad in (-8, 4, 1 << 41):
            s = [1 << 20, 1 << 10, 64] * 4
            s[i] = bad
            want = b.ATTN_ERR_ALIGN if i % 3 == 0 else b.ATTN_ERR_SHAPE       # one batch entry has no stride
            assert f(strides=arr(s), pos=OK + 2) == want, (i, bad)
    assert f(B=1 << 20, S=1 << 20) == b.ATTN_ERR_SHAPE and f(H_q=2 ** 31 - 1) == b.ATTN_ERR_SHAPE
    for n in ("q", "q_out", "k", "k_out"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    assert f(pos=OK + 2) == b.ATTN_ERR_ALIGN and f(freq=OK + 4) == b.ATTN_ERR_ALIGN


@pytest.mark.parametrize("entry", ["attn_cache_write", "attn_cache_write_f16", "attn_cache_read", "attn_cache_read_f16"])
def test_cache_refusals(b, entry):
    f = caller(b, entry, ROWS)
    for n in ("k", "v", "strides", "k_pages", "v_pages", "k_scale", "v_scale", "table", "start", "kv_len"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    assert f(kind=0, k_scale=None, v_scale=None, k=OK + 8) == b.ATTN_ERR_ALIGN
    for n in ("T", "B", "H_kv", "n_pages", "width"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    for D in (0, 32, 96, 512):
        assert f(D=D) == b.ATTN_ERR_UNSUPPORTED_D
    for size in (0, 8, 15, 24, 512, -16):
        assert f(page_size=size) == b.ATTN_ERR_UNSUPPORTED
    assert f(kind=2) == b.ATTN_ERR_UNSUPPORTED and f(kind=-1) == b.ATTN_ERR_UNSUPPORTED
    for i in range(4):
        for bad in (-8, 4, 1 << 41):
            s = [512, 64] * 2
            s[i] = bad
            assert f(strides=arr(s)) == b.ATTN_ERR_SHAPE
    assert f(width=1 << 27) == b.ATTN_ERR_SHAPE
    assert f(T=2 ** 31 - 1, H_kv=1 << 20) == b.ATTN_ERR_SHAPE and f(n_pages=2 ** 31 - 1, H_kv=1 << 10) == b.ATTN_ERR_SHAPE
    for n in ("k", "v", "k_pages", "v_pages", "k_scale", "v_scale"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    for n in ("table", "start", "kv_len"):
        assert f(**{n: OK + 2}) == b.ATTN_ERR_ALIGN


@pytest.mark.parametrize("suffix", ["", "_f16"])
def test_paged_refusals(b, suffix):
    f = caller(b, "attn_paged_fwd" + suffix, PAGED)
    for n in ("q", "strides", "o", "lse", "k_pages", "v_pages", "k_scale", "v_scale", "table", "start", "kv_len", "ws"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    for n in ("T", "B", "H_q", "H_kv", "n_pages", "width", "max_q"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    assert f(H_q=5) == b.ATTN_ERR_SHAPE and f(T=1 << 30) == b.ATTN_ERR_SHAPE and f(width=1 << 27) == b.ATTN_ERR_SHAPE
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
    for n in ("q", "o", "k_pages", "v_pages", "k_scale", "v_scale", "ws"):
        assert f(**{n: OK + 8}) == b.ATTN_ERR_ALIGN
    for n in ("lse", "table", "start", "kv_len"):
        assert f(**{n: OK + 2}) == b.ATTN_ERR_ALIGN
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert f(scale=s) == b.ATTN_ERR_SCALE
    need = b.attn_paged_fwd_workspace_bytes(3, 2, 4, 2, 64)
    assert need > 0 and f(ws_bytes=need - 1) == b.ATTN_ERR_WORKSPACE
    for bad in ((0, 1, 4, 2, 64), (3, 0, 4, 2, 64), (3, 2, 5, 2, 64), (3, 2, 4, 0, 64), (3, 2, 4, 2, 96), (1 << 30, 1, 4, 2, 64)):
        assert b.attn_paged_fwd_workspace_bytes(*bad) == -1


def test_the_binding_refuses_what_is_not_on_the_gpu_or_of_another_type(b):
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError):
        b.attn_rope(bf(1, 2, 3, 64), bf(1, 2, 3, 64), i32(1, 1, 3), torch.zeros(32, dtype=torch.float64), [32])
    with pytest.raises(TypeError):
        b.attn_cache_write(bf(3, 2, 64), bf(3, 2, 64), bf(4, 2, 16, 64), bf(4, 2, 16, 64), i32(1, 4), i32(2), i32(1))
    with pytest.raises(TypeError):
        b.attn_cache_read(bf(4, 2, 16, 64), bf(4, 2, 16, 64), i32(1, 4), i32(2), i32(1), 3)
    with pytest.raises(TypeError):
        b.attn_paged_fwd(bf(3, 2, 64), bf(4, 2, 16, 64), bf(4, 2, 16, 64), i32(1, 4), i32(2), i32(1))


def test_overlapping_output_rows_are_refused(b):
    x = torch.zeros(2, 3, 4, 8)
    b._check_output(x, "x")
    b._check_output(x.transpose(0, 2), "x")
    b._check_output(x[:, :, ::2], "x")
    b._check_output(x[:1].expand(1, 3, 4, 8), "x")
    for bad in (x[:1].expand(2, 3, 4, 8), x.as_strided((2, 3, 4, 8), (96, 24, 8, 1)), x.as_strided((3, 4, 8), (16, 4, 1))):
        with pytest.raises(ValueError):
            b._check_output(bad, "x")
