"""What attn_paged_tree refuses, on the host, before any HIP call (no GPU needed)."""
import pytest
import torch

from test_serving_abi import OK, PAGED, arr, b, caller  # noqa: F401

TREE = PAGED[:12] + [("mask", OK), ("words", 1)] + [x for x in PAGED[12:] if x[0] != "causal"]


@pytest.mark.parametrize("suffix", ["", "_f16"])
def test_tree_refusals(b, suffix):  # noqa: F811
    f = caller(b, "attn_paged_tree" + suffix, TREE)
    for n in ("q", "strides", "o", "lse", "k_pages", "v_pages", "k_scale", "v_scale", "table", "start", "kv_len", "ws", "mask"):
        assert f(**{n: None}) == b.ATTN_ERR_NULL
    for n in ("T", "B", "H_q", "H_kv", "n_pages", "width", "max_q", "words"):
        assert f(**{n: 0}) == b.ATTN_ERR_SHAPE and f(**{n: -1}) == b.ATTN_ERR_SHAPE
    assert f(words=1025) == b.ATTN_ERR_SHAPE and f(words=1024, start=OK + 2) == b.ATTN_ERR_ALIGN
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
    assert f(mask=OK + 4) == b.ATTN_ERR_ALIGN
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert f(scale=s) == b.ATTN_ERR_SCALE
    need = b.attn_paged_tree_workspace_bytes(3, 2, 4, 2, 64)
    assert need > 0 and f(ws_bytes=need - 1) == b.ATTN_ERR_WORKSPACE
    for bad in ((0, 1, 4, 2, 64), (3, 0, 4, 2, 64), (3, 2, 5, 2, 64), (3, 2, 4, 0, 64), (3, 2, 4, 2, 96), (1 << 30, 1, 4, 2, 64),
                (3, (1 << 30) + 1, 4, 2, 64)):
        assert b.attn_paged_tree_workspace_bytes(*bad) == -1
    for B in ((1 << 30) + 1, 2 ** 31 - 64, 2 ** 31 - 1):
        assert f(B=B, start=OK + 2) == b.ATTN_ERR_SHAPE
    many = dict(T=1 << 22, B=1 << 22, H_q=8, H_kv=8, strides=arr([512, 64]))
    assert f(**many) == b.ATTN_ERR_SHAPE


def test_the_binding_refuses_what_is_not_on_the_gpu(b):  # noqa: F811
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError):
        b.attn_paged_tree(bf(3, 2, 64), bf(4, 2, 16, 64), bf(4, 2, 16, 64), i32(1, 4), i32(2), i32(1), torch.zeros(3, 1, dtype=torch.int64))
