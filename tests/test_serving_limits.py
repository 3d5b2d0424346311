"""The largest calls of the serving entry points, and what a refusal says, on the host (no GPU needed)."""
import ctypes

import pytest
import torch

from test_serving_abi import OK, PAGED, ROPE, ROWS, arr, b, caller  # noqa: F401


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf")])
def test_a_refused_scale_is_explained(b, scale):  # noqa: F811
    """attn_paged_fwd refuses a scale of 0, and the status text may not call that one fine."""
    assert caller(b, "attn_paged_fwd", PAGED)(scale=scale) == b.ATTN_ERR_SCALE
    text = b.attn_strerror(b.ATTN_ERR_SCALE)
    assert "> 0" in text and ">= 0" not in text


@pytest.mark.parametrize("entry, spec", [("attn_cache_write", ROWS), ("attn_cache_read_f16", ROWS), ("attn_paged_fwd", PAGED),
                                         ("attn_paged_fwd_f16", PAGED)])
def test_a_batch_that_the_lanes_cannot_count_is_refused(b, entry, spec):  # noqa: F811
    """The kernels step through the sequences by up to 1024 at a time: with B next to 2^31 the step's sum is negative, below B, and
    an index in front of kv_len.  (Arguments that are misaligned as well, so that nothing could be launched.)"""
    f = caller(b, entry, spec)
    for B in ((1 << 30) + 1, 2 ** 31 - 1025, 2 ** 31 - 64, 2 ** 31 - 2, 2 ** 31 - 1):
        assert f(B=B, start=OK + 2) == b.ATTN_ERR_SHAPE
        assert b.attn_paged_fwd_workspace_bytes(3, B, 4, 2, 64) == -1
    assert f(B=1 << 30, start=OK + 2) == b.ATTN_ERR_ALIGN
    assert b.attn_paged_fwd_workspace_bytes(3, 1 << 30, 4, 2, 64) > 0


@pytest.mark.parametrize("suffix", ["", "_f16"])
def test_launches_of_too_many_threads_are_refused_before_any(b, suffix):  # noqa: F811
    """The runtime takes less than 2^32 threads in a dimension: a call that needs more is refused with its arguments, not by one of
    its launches (of which attention has up to three)."""
    rope = caller(b, "attn_rope" + suffix, ROPE)
    one = dict(H_kv=0, H_q=1, S=1 << 30, n_axes=1, sections=arr([32], ctypes.c_int), strides=arr([0, 0, 64] * 4))
    assert rope(**one) == b.ATTN_ERR_SHAPE                                        # 2^24 workgroups of 256 threads
    for entry in ("attn_cache_write", "attn_cache_read"):
        rows = caller(b, entry + suffix, ROWS)
        assert rows(T=1 << 29, H_kv=1, strides=arr([64, 0] * 2)) == b.ATTN_ERR_SHAPE
    paged = caller(b, "attn_paged_fwd" + suffix, PAGED)
    many = dict(T=1 << 22, B=1 << 22, H_q=8, H_kv=8, strides=arr([512, 64]))
    assert paged(**many) == b.ATTN_ERR_SHAPE                                      # a row workgroup for every sequence and head
    merge = dict(T=(1 << 26) - 1, B=1, H_q=8, H_kv=8, D=256, max_q=1 << 26, width=64, strides=arr([2048, 256]))
    assert paged(**merge) == b.ATTN_ERR_SHAPE                                     # tiles: as many workgroups as run at once; the merge: 2^27


def test_rows_that_a_c_int_cannot_count_are_refused(b):  # noqa: F811
    """A view that repeats one row 2^32 + 1 times is a legal input of attn_cache_write; handed on in 32 bits it would be one row."""
    class Rows:
        dtype, is_cuda, device = torch.bfloat16, True, torch.device("cuda", 0)

        def __init__(self, t):
            self.shape, self.stride, self.dim = t.shape, t.stride, t.dim
    fine = torch.zeros(1, 1, 64, dtype=torch.bfloat16)
    b._check_rows(Rows(fine.expand(2 ** 31 - 1, 1, 64)), torch.bfloat16, 3, "k", Rows.device)
    for n in (2 ** 31, 2 ** 32 + 1):
        with pytest.raises(ValueError):
            b._check_rows(Rows(fine.expand(n, 1, 64)), torch.bfloat16, 3, "k", Rows.device)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_the_workspace_follows_the_rows_of_the_call(b, D):  # noqa: F811
    """Partial rows for as many units as run at once, in tiles that the call's rows can need: a single token of four query heads to
    a key head does not pay for tiles of 64 rows.  (1088 slots; tiles of 16 rows up to 16, 32 up to 32, then 64, but 32 at D = 256.)"""
    need = lambda T, B=1, G=1: b.attn_paged_fwd_workspace_bytes(T, B, 2 * G, 2, D)
    slots = lambda rows: 1088 * rows * (D + 1) * 4
    assert need(1, 1, 4) == slots(16) + 16 and need(4, 4, 4) == slots(16) + 4 * 16
    assert need(17) == slots(32) + 17 * 16 and need(8, 1, 4) == slots(32) + 8 * 16
    assert need(33) == slots(32 if D == 256 else 64) + 33 * 16
    most = 64 if D == 256 else 128
    assert need(most) == slots(most // 2) + most * 16
    assert need(most + 1) == slots(most // 2) + slots(2 * most) + (most + 1) * 16      # the tile kernels too
    sizes = [need(T, 1, G) for G in (1, 4) for T in range(1, 300)]
    assert sizes[:299] == sorted(sizes[:299]) and sizes[299:] == sorted(sizes[299:])
