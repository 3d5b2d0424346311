"""Binding of libmi355attn.so: argument marshalling only.

Same names as include/attn_fwd.h.  There is no fallback: importing this module
raises if the library has not been built (python -m paper_2512_18134_amd.build).
PyTorch appears only as the owner of device memory and of the stream.

A call on plain contiguous tensors goes through the extension module _marshal
(csrc/marshal.cpp), which is loaded on the first call; it hands every other call
back, and the code here checks its arguments, raises what is to be raised and calls
the library through ctypes.  Where the module was not built (no torch at build time)
every call goes that way: the same kernels, some 10 us more of host work.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# ATTN_FWD_LIB (debug only) loads another build of the same library, e.g. a schedule experiment
LIB_PATH = os.environ.get("ATTN_FWD_LIB", os.path.join(_HERE, "libmi355attn.so"))

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libmi355attn.so is not built: run `python -m paper_2512_18134_amd.build` "
        "(there is no CPU or PyTorch fallback for attn_fwd)")

_lib = ctypes.CDLL(LIB_PATH)
_lib.attn_fwd.restype = ctypes.c_int
_lib.attn_fwd.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
_lib.attn_fwd_f16.restype = ctypes.c_int
_lib.attn_fwd_f16.argtypes = _lib.attn_fwd.argtypes
_lib.attn_fwd_splitkv.restype = ctypes.c_int
_lib.attn_fwd_splitkv.argtypes = ([ctypes.c_void_p] * 6 + [ctypes.c_longlong, ctypes.c_int] + [ctypes.c_int] * 6
                                  + [ctypes.c_float, ctypes.c_void_p])
_lib.attn_fwd_splitkv_f16.restype = ctypes.c_int
_lib.attn_fwd_splitkv_f16.argtypes = _lib.attn_fwd_splitkv.argtypes
_lib.attn_fwd_splitkv_workspace_bytes.restype = ctypes.c_longlong
_lib.attn_fwd_splitkv_workspace_bytes.argtypes = [ctypes.c_int] * 5
_lib.attn_bwd.restype = ctypes.c_int
_lib.attn_bwd.argtypes = [ctypes.c_void_p] * 10 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
_lib.attn_bwd_f16.restype = ctypes.c_int
_lib.attn_bwd_f16.argtypes = _lib.attn_bwd.argtypes
_lib.attn_bwd_noalloc.restype = ctypes.c_int
_lib.attn_bwd_noalloc.argtypes = [ctypes.c_void_p] * 9 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
_lib.attn_strerror.restype = ctypes.c_char_p
_lib.attn_strerror.argtypes = [ctypes.c_int]
_lib.attn_version.restype = ctypes.c_int
_lib.attn_version.argtypes = []
_lib.attn_workgroup_tile.restype = ctypes.c_int
_lib.attn_workgroup_tile.argtypes = [ctypes.c_int] * 4 + [ctypes.c_longlong] + [ctypes.POINTER(ctypes.c_int)] * 2

ATTN_OK = 0
ATTN_ERR_NULL = -1
ATTN_ERR_SHAPE = -2
ATTN_ERR_UNSUPPORTED_D = -3
ATTN_ERR_ALIGN = -4
ATTN_ERR_SCALE = -5
ATTN_ERR_LAUNCH = -6
ATTN_ERR_UNSUPPORTED = -7
ATTN_ERR_WORKSPACE = -8


class AttnError(RuntimeError):
    def __init__(self, status):
        self.status = status
        super().__init__("attn_fwd: %s (status %d)" % (attn_strerror(status), status))


def attn_strerror(status):
    return _lib.attn_strerror(int(status)).decode()


def attn_version():
    return int(_lib.attn_version())


_lib.attn_workgroup_queue_entry.restype = ctypes.c_int
_lib.attn_workgroup_queue_entry.argtypes = [ctypes.c_int] * 4 + [ctypes.POINTER(ctypes.c_int)]


def attn_workgroup_queue_entry(workgroup, n_workgroups, n_entries, pass_):
    """Host-side view of the persistent forward launch: the queue entry workgroup `workgroup` takes up in pass
    `pass_`, or -1."""
    entry = ctypes.c_int(-2)
    rc = int(_lib.attn_workgroup_queue_entry(int(workgroup), int(n_workgroups), int(n_entries), int(pass_),
                                             ctypes.byref(entry)))
    if rc != ATTN_OK:
        raise AttnError(rc)
    return entry.value


def attn_workgroup_tile(causal, workgroup, n_heads, n_tiles, head_bytes=0):
    """attn_workgroup_tile (host-only diagnostic): the (head, tile) that workgroup id works on."""
    head, tile = ctypes.c_int(-1), ctypes.c_int(-1)
    rc = int(_lib.attn_workgroup_tile(int(bool(causal)), int(workgroup), int(n_heads), int(n_tiles), int(head_bytes),
                                      ctypes.byref(head), ctypes.byref(tile)))
    if rc != ATTN_OK:
        raise AttnError(rc)
    return head.value, tile.value


MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")
_marshal_module = None


class _NotBuilt:
    """In place of the extension module: every call is handed back."""
    fwd = splitkv = bwd = rope = write = read = paged = staticmethod(lambda *args: None)


def _native():
    """The extension module, loaded on first use (it needs torch's libraries in the process)."""
    global _marshal_module
    if _marshal_module is None and not os.path.exists(MARSHAL_PATH):
        _marshal_module = _NotBuilt
    if _marshal_module is None:
        import torch
        from . import _marshal as module
        address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
        module.set_entries(address(_lib.attn_fwd), address(_lib.attn_fwd_f16), address(_lib.attn_fwd_splitkv),
                           address(_lib.attn_fwd_splitkv_f16), address(_lib.attn_bwd), address(_lib.attn_bwd_f16),
                           address(_lib.attn_fwd_splitkv_workspace_bytes),
                           getattr(torch._C, "_cuda_getCurrentRawStream",
                                   lambda index: torch.cuda.current_stream(index).cuda_stream))
        module.set_serving_entries(*(address(getattr(_lib, name + suffix))
                                     for name in ("attn_rope", "attn_cache_write", "attn_cache_read", "attn_paged_fwd")
                                     for suffix in ("", "_f16")), address(_lib.attn_paged_fwd_workspace_bytes))
        _marshal_module = module
    return _marshal_module


def _finish(result):
    """What a native call returned: its outputs, or a status to raise."""
    if type(result) is tuple:
        return result
    raise AttnError(result)


def attn_fwd_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_fwd(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S_q, S_kv, D,
                             int(bool(causal)), float(scale), stream_ptr))


def attn_fwd_f16_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """attn_fwd_f16 with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_fwd_f16(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, H, S_q, S_kv, D,
                                 int(bool(causal)), float(scale), stream_ptr))


def attn_fwd(q, k, v, o=None, lse=None, causal=False, scale=None, stream=None):
    """attn_fwd on torch device tensors.

    q [B,H,S_q,D], k/v [B,H,S_kv,D]: contiguous bf16 on the GPU.  o (bf16) and
    lse (fp32 [B,H,S_q]) are allocated when not given.  The launch goes to
    `stream` (default: torch's current stream) and is asynchronous.  What a call
    with another stream allocates belongs to that stream; tensors that the caller
    passes have to outlive the call's kernels (Tensor.record_stream), as with
    any operation on a stream that is not the tensor's own.
    Returns (o, lse).
    """
    r = (_marshal_module or _native()).fwd(0, q, k, v, o, lse, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal(attn_fwd_raw, torch.bfloat16, q, k, v, o, lse, causal, scale, stream)


def attn_fwd_f16(q, k, v, o=None, lse=None, causal=False, scale=None, stream=None):
    """attn_fwd_f16 on torch device tensors: as attn_fwd, with fp16 q, k, v, o (D = 64 or 128)."""
    r = (_marshal_module or _native()).fwd(1, q, k, v, o, lse, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal(attn_fwd_f16_raw, torch.float16, q, k, v, o, lse, causal, scale, stream)


def _allocate(make, device, stream, returned=True):
    """A call's own allocation, made on the stream that its kernels run on: the caching allocator then gives the memory
    to nobody else before they are done, and gives them none that kernels of another stream still use.  What is
    returned to the caller may be used on the caller's current stream as well until it is freed."""
    import torch

    if stream is None:
        return make()
    current = torch.cuda.current_stream(device)
    if stream.cuda_stream == current.cuda_stream:
        return make()
    if not isinstance(stream, torch.cuda.Stream):
        stream = (torch.cuda.ExternalStream(stream.cuda_stream, device=device) if stream.cuda_stream else
                  torch.cuda.default_stream(device))
    with torch.cuda.stream(stream):
        t = make()
    if returned:
        t.record_stream(current)
    return t


def _marshal(entry, dt, q, k, v, o, lse, causal, scale, stream):
    import torch

    for t in (q, k, v):
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("q, k, v must be contiguous 4-D %s tensors on the GPU" % dt)
    B, H, S_q, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[1] != H or k.shape[3] != D:
        raise ValueError("q, k, v shapes do not agree")
    S_kv = k.shape[2]
    if o is None:
        o = _allocate(lambda: torch.empty_like(q), q.device, stream)
    if lse is None:
        lse = _allocate(lambda: torch.empty((B, H, S_q), dtype=torch.float32, device=q.device), q.device, stream)
    if o.dtype != dt or o.shape != q.shape or not o.is_contiguous() or not o.is_cuda:
        raise TypeError("o must be a contiguous GPU tensor shaped and typed like q")
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, S_q) or not lse.is_contiguous() or not lse.is_cuda:
        raise TypeError("lse must be a contiguous fp32 GPU tensor [B,H,S_q]")
    if scale is None:
        scale = 1.0 / float(D) ** 0.5
    if stream is None:
        stream = torch.cuda.current_stream(q.device)
    with torch.cuda.device(q.device):
        rc = entry(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                   B, H, S_q, S_kv, D, causal, scale, stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)
    return o, lse


def attn_bwd_raw(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr, ws_ptr,
                 B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point attn_bwd with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_bwd(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr, ws_ptr,
                             B, H, S_q, S_kv, D, int(bool(causal)), float(scale), stream_ptr))


def attn_bwd_f16_raw(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr, ws_ptr,
                     B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point attn_bwd_f16 with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_bwd_f16(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr, ws_ptr,
                                 B, H, S_q, S_kv, D, int(bool(causal)), float(scale), stream_ptr))


def attn_bwd_noalloc_raw(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr,
                         B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point attn_bwd_noalloc with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_bwd_noalloc(q_ptr, k_ptr, v_ptr, o_ptr, do_ptr, lse_ptr, dq_ptr, dk_ptr, dv_ptr,
                                     B, H, S_q, S_kv, D, int(bool(causal)), float(scale), stream_ptr))


def attn_bwd_noalloc(q, k, v, o, d_o, lse, dq, dk, dv, causal=False, scale=None, stream=None):
    """attn_bwd_noalloc on torch device tensors: attn_bwd with the library's own workspace.  The caller
    passes every output (this wrapper allocates nothing either).  Returns (dq, dk, dv)."""
    import torch
    entry = lambda *a: attn_bwd_noalloc_raw(*(a[:9] + a[10:]))   # drop the workspace address
    return _marshal_bwd(entry, torch.bfloat16, q, k, v, o, d_o, lse, dq, dk, dv, False, causal, scale, stream)


def attn_bwd_f16(q, k, v, o, d_o, lse, dq=None, dk=None, dv=None, delta_ws=None, causal=False, scale=None,
                 stream=None):
    """attn_bwd_f16 on torch device tensors: as attn_bwd, with fp16 tensors."""
    r = (_marshal_module or _native()).bwd(1, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_bwd(attn_bwd_f16_raw, torch.float16, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale,
                        stream)


def attn_bwd(q, k, v, o, d_o, lse, dq=None, dk=None, dv=None, delta_ws=None, causal=False, scale=None, stream=None):
    """attn_bwd on torch device tensors (include/attn_bwd.h).

    q, o, d_o [B,H,S_q,D], k, v [B,H,S_kv,D]: contiguous bf16 on the GPU; lse fp32 [B,H,S_q] as
    written by attn_fwd.  dq, dk, dv (bf16) and the fp32 workspace delta_ws (2*B*H*S_q floats) are
    allocated when not given.  Asynchronous on `stream`.  Returns (dq, dk, dv).
    """
    r = (_marshal_module or _native()).bwd(0, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_bwd(attn_bwd_raw, torch.bfloat16, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale, stream)


def _marshal_bwd(entry, dt, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale, stream):
    import torch

    for t in (q, k, v, o, d_o):
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("q, k, v, o, d_o must be contiguous 4-D %s tensors on the GPU" % dt)
    B, H, S_q, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[1] != H or k.shape[3] != D:
        raise ValueError("q, k, v shapes do not agree")
    if o.shape != q.shape or d_o.shape != q.shape:
        raise ValueError("o and d_o must be shaped like q")
    S_kv = k.shape[2]
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, S_q) or not lse.is_contiguous() or not lse.is_cuda:
        raise TypeError("lse must be a contiguous fp32 GPU tensor [B,H,S_q]")
    no_ws = delta_ws is False          # attn_bwd_noalloc: the library's own workspace, outputs from the caller
    if no_ws and (dq is None or dk is None or dv is None):
        raise TypeError("attn_bwd_noalloc: the caller passes dq, dk, dv")
    dq = _allocate(lambda: torch.empty_like(q), q.device, stream) if dq is None else dq
    dk = _allocate(lambda: torch.empty_like(k), q.device, stream) if dk is None else dk
    dv = _allocate(lambda: torch.empty_like(v), q.device, stream) if dv is None else dv
    if delta_ws is None:
        delta_ws = _allocate(lambda: torch.empty((2, B, H, S_q), dtype=torch.float32, device=q.device), q.device, stream,
                             returned=False)
    for t, like in ((dq, q), (dk, k), (dv, v)):
        if t.dtype != dt or t.shape != like.shape or not t.is_contiguous() or not t.is_cuda:
            raise TypeError("dq, dk, dv must be contiguous GPU tensors shaped and typed like q, k, v")
    if not no_ws and (delta_ws.dtype != torch.float32 or delta_ws.numel() < 2 * B * H * S_q
                      or not delta_ws.is_contiguous() or not delta_ws.is_cuda):
        raise TypeError("delta_ws must be a contiguous fp32 GPU tensor with at least 2*B*H*S_q elements")
    if scale is None:
        scale = 1.0 / float(D) ** 0.5
    if stream is None:
        stream = torch.cuda.current_stream(q.device)
    with torch.cuda.device(q.device):
        rc = entry(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), d_o.data_ptr(), lse.data_ptr(),
                   dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), 0 if no_ws else delta_ws.data_ptr(),
                   B, H, S_q, S_kv, D, causal, scale, stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)
    return dq, dk, dv


def attn_fwd_splitkv_workspace_bytes(B, H, S_q, D, n_split):
    return int(_lib.attn_fwd_splitkv_workspace_bytes(B, H, S_q, D, n_split))


def attn_fwd_splitkv_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, ws_ptr, ws_bytes, n_split,
                         B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point attn_fwd_splitkv with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_fwd_splitkv(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, ws_ptr, ws_bytes, n_split,
                                     B, H, S_q, S_kv, D, int(bool(causal)), float(scale), stream_ptr))


def attn_fwd_splitkv_f16_raw(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, ws_ptr, ws_bytes, n_split,
                             B, H, S_q, S_kv, D, causal, scale, stream_ptr):
    """The C entry point attn_fwd_splitkv_f16 with raw integer addresses; returns the attn_status."""
    return int(_lib.attn_fwd_splitkv_f16(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, ws_ptr, ws_bytes, n_split,
                                         B, H, S_q, S_kv, D, int(bool(causal)), float(scale), stream_ptr))


def attn_fwd_splitkv(q, k, v, n_split, o=None, lse=None, workspace=None, causal=False, scale=None, stream=None):
    """attn_fwd_splitkv on torch device tensors (bf16).  `workspace`: a contiguous GPU tensor of at least
    attn_fwd_splitkv_workspace_bytes(...) bytes (allocated when not given).  Returns (o, lse)."""
    r = (_marshal_module or _native()).splitkv(0, q, k, v, n_split, o, lse, workspace, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_splitkv(attn_fwd_splitkv_raw, torch.bfloat16, q, k, v, n_split, o, lse, workspace, causal, scale,
                            stream)


def attn_fwd_splitkv_f16(q, k, v, n_split, o=None, lse=None, workspace=None, causal=False, scale=None, stream=None):
    """attn_fwd_splitkv_f16 on torch device tensors: as attn_fwd_splitkv, with fp16 tensors."""
    r = (_marshal_module or _native()).splitkv(1, q, k, v, n_split, o, lse, workspace, causal, scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_splitkv(attn_fwd_splitkv_f16_raw, torch.float16, q, k, v, n_split, o, lse, workspace, causal, scale,
                            stream)


def _marshal_splitkv(entry, dt, q, k, v, n_split, o, lse, workspace, causal, scale, stream):
    import torch

    for t in (q, k, v):
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("q, k, v must be contiguous 4-D %s tensors on the GPU" % dt)
    B, H, S_q, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[1] != H or k.shape[3] != D:
        raise ValueError("q, k, v shapes do not agree")
    S_kv = k.shape[2]
    o = _allocate(lambda: torch.empty_like(q), q.device, stream) if o is None else o
    if lse is None:
        lse = _allocate(lambda: torch.empty((B, H, S_q), dtype=torch.float32, device=q.device), q.device, stream)
    if o.dtype != dt or o.shape != q.shape or not o.is_contiguous() or not o.is_cuda:
        raise TypeError("o must be a contiguous GPU tensor shaped and typed like q")
    if lse.dtype != torch.float32 or tuple(lse.shape) != (B, H, S_q) or not lse.is_contiguous() or not lse.is_cuda:
        raise TypeError("lse must be a contiguous fp32 GPU tensor [B,H,S_q]")
    need = attn_fwd_splitkv_workspace_bytes(B, H, S_q, D, n_split)
    if workspace is None:
        workspace = _allocate(lambda: torch.empty((max(need, 16),), dtype=torch.uint8, device=q.device), q.device, stream,
                              returned=False)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous GPU tensor")
    if scale is None:
        scale = 1.0 / float(D) ** 0.5
    if stream is None:
        stream = torch.cuda.current_stream(q.device)
    with torch.cuda.device(q.device):
        rc = entry(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), n_split,
                   B, H, S_q, S_kv, D, causal, scale, stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)
    return o, lse


# ---------------------------------------------------------------------------------------------------------------------
# Rotary positions, the paged cache and attention over it (include/attn_rope.h, include/attn_cache.h)

ATTN_CACHE_16BIT = 0
ATTN_CACHE_E4M3 = 1

_INT_MAX = 2 ** 31 - 1
_pointer, _int, _int64, _float = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float
for _name, _args in (("attn_rope", [_pointer] * 8 + [_int] * 8 + [_pointer]),
                     ("attn_cache_write", [_pointer] * 10 + [_int] * 8 + [_pointer]),
                     ("attn_cache_read", [_pointer] * 10 + [_int] * 8 + [_pointer]),
                     ("attn_paged_fwd", [_pointer] * 11 + [_int, _pointer, _int64, _int] + [_int] * 9 + [_float, _pointer])):
    for _suffix in ("", "_f16"):
        getattr(_lib, _name + _suffix).restype = _int
        getattr(_lib, _name + _suffix).argtypes = _args
_lib.attn_paged_fwd_workspace_bytes.restype = _int64
_lib.attn_paged_fwd_workspace_bytes.argtypes = [_int] * 5


def _strides(*dims):
    """A C array of the strides of (tensor, dimension) pairs; a dimension of one element has none."""
    return (_int64 * len(dims))(*(t.stride(d) if t is not None and t.shape[d] > 1 else 0 for t, d in dims))


def _check_rows(t, dt, dims, name, device):
    """Rows of contiguous elements, any strides between them."""
    if t.dtype != dt or not t.is_cuda or t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise TypeError("%s must be a %d-D %s tensor on the GPU whose last dimension is contiguous" % (name, dims, dt))
    if max(t.shape) > _INT_MAX:                       # (a broadcast view may be; ctypes would keep 32 bits of it)
        raise ValueError("%s has a dimension beyond 2^31 - 1" % name)
    if t.device != device:
        raise ValueError("%s is on another device" % name)


def _check_output(t, name):
    """Two rows of an output must not share memory: sorted by stride, every dimension steps over the ones below it."""
    reach = 1
    for stride, size in sorted((t.stride(d), t.shape[d]) for d in range(t.dim()) if t.shape[d] > 1):
        if stride < reach:
            raise ValueError("rows of %s overlap" % name)
        reach = stride * (size - 1) + reach


def _check_array(t, dtype, shape, name, device):
    if t.dtype != dtype or not t.is_cuda or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s GPU tensor of shape %s" % (name, dtype, tuple(shape)))
    if t.device != device:
        raise ValueError("%s is on another device" % name)


def _address(t):
    return None if t is None else t.data_ptr()


def attn_rope(q, k, pos, freq, sections, q_out=None, k_out=None, interleaved=False, inverse=False, stream=None):
    """attn_rope on torch device tensors (include/attn_rope.h): q and k turned by the positions of their tokens.

    q [B,H_q,S,D], k [B,H_kv,S,D] (or None): bf16 on the GPU, D contiguous elements, other strides in multiples of 8, so slices
    of a projection's rows are fine (rows[:, :H_q].transpose(0, 1)[None]).  pos int32 [n_axes,B,S], freq fp64 [pairs], radians
    per unit of position; sections: how many pairs follow each axis (sum = pairs; 2 * pairs of a head's D elements are
    turned, the others are copied).  q_out and k_out are allocated when not given (contiguous); they may be q and k.
    inverse=True turns back: with the gradients of the outputs in place of q and k it gives the gradients of the inputs.
    Asynchronous on `stream`.  Returns (q_out, k_out).
    """
    r = (_marshal_module or _native()).rope(0, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_rope(_lib.attn_rope, torch.bfloat16, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream)


def attn_rope_f16(q, k, pos, freq, sections, q_out=None, k_out=None, interleaved=False, inverse=False, stream=None):
    """attn_rope_f16 on torch device tensors: as attn_rope, with fp16 tensors."""
    r = (_marshal_module or _native()).rope(1, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_rope(_lib.attn_rope_f16, torch.float16, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream)


def _marshal_rope(entry, dt, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream):
    import torch

    _check_rows(q, dt, 4, "q", q.device)
    B, H_q, S, D = q.shape
    H_kv = 0
    if k is not None:
        _check_rows(k, dt, 4, "k", q.device)
        H_kv = k.shape[1]
        if k.shape[0] != B or k.shape[2] != S or k.shape[3] != D:
            raise ValueError("q, k shapes do not agree")
    elif k_out is not None:
        raise ValueError("k_out without k")
    sections = [int(n) for n in sections]
    _check_array(pos, torch.int32, (len(sections), B, S), "pos", q.device)
    _check_array(freq, torch.float64, (sum(sections),), "freq", q.device)
    if q_out is None:
        q_out = _allocate(lambda: torch.empty(q.shape, dtype=dt, device=q.device), q.device, stream)
    if k_out is None and k is not None:
        k_out = _allocate(lambda: torch.empty(k.shape, dtype=dt, device=q.device), q.device, stream)
    for t, like, name in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        if t is None:
            continue
        _check_rows(t, dt, 4, name, q.device)
        if t.shape != like.shape:
            raise ValueError("%s is not shaped like its input" % name)
        _check_output(t, name)
    if stream is None:
        stream = torch.cuda.current_stream(q.device)
    strides = _strides(*((t, d) for t in (q, q_out, k, k_out) for d in range(3)))
    with torch.cuda.device(q.device):
        rc = entry(q.data_ptr(), q_out.data_ptr(), _address(k), _address(k_out), strides, pos.data_ptr(), freq.data_ptr(),
                   (_int * len(sections))(*sections), len(sections), B, H_q, H_kv, S, D, int(bool(interleaved)),
                   int(bool(inverse)), stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)
    return q_out, k_out


def _check_cache(dt, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, device):
    """The cache's tensors; returns (kind, n_pages, H_kv, page_size, D, B, table_width)."""
    import torch

    if k_pages.dim() != 4:
        raise TypeError("k_pages must be [n_pages, H_kv, page_size, D]")
    kind = ATTN_CACHE_E4M3 if k_pages.dtype == torch.float8_e4m3fn else ATTN_CACHE_16BIT
    pages_dt = torch.float8_e4m3fn if kind == ATTN_CACHE_E4M3 else dt
    _check_array(k_pages, pages_dt, k_pages.shape, "k_pages", device)
    _check_array(v_pages, pages_dt, k_pages.shape, "v_pages", device)
    if kind == ATTN_CACHE_E4M3:
        if k_scale is None or v_scale is None:
            raise TypeError("an e4m3 cache needs k_scale and v_scale")
        _check_array(k_scale, torch.uint8, k_pages.shape[:3], "k_scale", device)
        _check_array(v_scale, torch.uint8, k_pages.shape[:3], "v_scale", device)
    elif k_scale is not None or v_scale is not None:
        raise TypeError("a 16-bit cache has no scales")
    if page_table.dim() != 2:
        raise TypeError("page_table must be [B, table_width]")
    B = page_table.shape[0]
    _check_array(page_table, torch.int32, page_table.shape, "page_table", device)
    _check_array(start, torch.int32, (B + 1,), "start", device)
    _check_array(kv_len, torch.int32, (B,), "kv_len", device)
    n_pages, H_kv, page_size, D = k_pages.shape
    return kind, n_pages, H_kv, page_size, D, B, page_table.shape[1]


def attn_cache_write(k, v, k_pages, v_pages, page_table, start, kv_len, k_scale=None, v_scale=None, stream=None):
    """attn_cache_write on torch device tensors (include/attn_cache.h): new rows of K and V into their pages.

    k, v [T,H_kv,D] bf16, D contiguous elements, other strides in multiples of 8.  k_pages, v_pages [n_pages,H_kv,page_size,D]: bf16, or
    float8_e4m3fn with k_scale, v_scale uint8 [n_pages,H_kv,page_size].  page_table int32 [B,table_width], start int32 [B+1],
    kv_len int32 [B]: rows start[b] .. start[b+1]-1 become the last positions below kv_len[b] of sequence b.
    Asynchronous on `stream`.  Returns (k_pages, v_pages).
    """
    r = (_marshal_module or _native()).write(0, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    _marshal_rows(_lib.attn_cache_write, torch.bfloat16, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale,
                  stream)
    return k_pages, v_pages


def attn_cache_write_f16(k, v, k_pages, v_pages, page_table, start, kv_len, k_scale=None, v_scale=None, stream=None):
    """attn_cache_write_f16 on torch device tensors: as attn_cache_write, with fp16 rows (and fp16 or e4m3 pages)."""
    r = (_marshal_module or _native()).write(1, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, stream)
    if r is not None:
        return _finish(r)
    import torch
    _marshal_rows(_lib.attn_cache_write_f16, torch.float16, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale,
                  stream)
    return k_pages, v_pages


def attn_cache_read(k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale=None, v_scale=None, k=None, v=None,
                    stream=None):
    """attn_cache_read on torch device tensors (include/attn_cache.h): the last positions below kv_len[b] of sequence b into
    rows start[b] .. start[b+1]-1 of k and v, [n_rows,H_kv,D] bf16, allocated when not given (D contiguous elements,
    other strides in multiples of 8: [H_kv,n_rows,D] tensors transposed are what attn_fwd takes).  Rows of no sequence are left as they were.  The
    cache's arguments are those of attn_cache_write.  Asynchronous on `stream`.  Returns (k, v).
    """
    r = (_marshal_module or _native()).read(0, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale, k, v,
                                            stream)
    if r is not None:
        return _finish(r)
    import torch
    return _read(_lib.attn_cache_read, torch.bfloat16, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale, k,
                 v, stream)


def attn_cache_read_f16(k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale=None, v_scale=None, k=None, v=None,
                        stream=None):
    """attn_cache_read_f16 on torch device tensors: as attn_cache_read, with fp16 rows."""
    r = (_marshal_module or _native()).read(1, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale, k, v,
                                            stream)
    if r is not None:
        return _finish(r)
    import torch
    return _read(_lib.attn_cache_read_f16, torch.float16, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale,
                 k, v, stream)


def _read(entry, dt, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale, k, v, stream):
    import torch

    shape = (int(n_rows), k_pages.shape[1], k_pages.shape[3])
    make = lambda: torch.empty(shape, dtype=dt, device=k_pages.device)
    k = _allocate(make, k_pages.device, stream) if k is None else k
    v = _allocate(make, k_pages.device, stream) if v is None else v
    for t, name in ((k, "k"), (v, "v")):
        if tuple(t.shape) != shape:
            raise ValueError("%s must be [n_rows, H_kv, D]" % name)
        _check_output(t, name)
    _marshal_rows(entry, dt, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, stream)
    return k, v


def _marshal_rows(entry, dt, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, stream):
    import torch

    _check_rows(k, dt, 3, "k", k.device)
    _check_rows(v, dt, 3, "v", k.device)
    kind, n_pages, H_kv, page_size, D, B, width = _check_cache(dt, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale,
                                                               k.device)
    if k.shape != v.shape or tuple(k.shape[1:]) != (H_kv, D):
        raise ValueError("k, v must be [T, H_kv, D] with the cache's heads")
    if stream is None:
        stream = torch.cuda.current_stream(k.device)
    with torch.cuda.device(k.device):
        rc = entry(k.data_ptr(), v.data_ptr(), _strides((k, 0), (k, 1), (v, 0), (v, 1)), k_pages.data_ptr(), v_pages.data_ptr(),
                   _address(k_scale), _address(v_scale), page_table.data_ptr(), start.data_ptr(), kv_len.data_ptr(), kind,
                   k.shape[0], B, H_kv, D, n_pages, page_size, width, stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)


def attn_paged_fwd_workspace_bytes(T, B, H_q, H_kv, D):
    return int(_lib.attn_paged_fwd_workspace_bytes(T, B, H_q, H_kv, D))


def attn_paged_fwd(q, k_pages, v_pages, page_table, start, kv_len, k_scale=None, v_scale=None, o=None, lse=None, workspace=None,
                   causal=True, scale=None, max_q=None, stream=None):
    """attn_paged_fwd on torch device tensors (include/attn_cache.h): the new tokens' queries against the cache.

    q [T,H_q,D] bf16, D contiguous elements, other strides in multiples of 8; H_q a multiple of the cache's H_kv.  The cache's arguments are
    those of attn_cache_write, which has put the same rows' keys and values there.  o (bf16 [T,H_q,D]) and lse (fp32 [T,H_q])
    are allocated when not given; rows of no sequence are left as they were.  workspace: a contiguous GPU tensor of at least
    attn_paged_fwd_workspace_bytes(...) bytes (allocated when not given); calls that overlap in time need one each.
    causal: row i of n_b sees the keys up to its own position, otherwise all kv_len[b] of them.  max_q: the largest n_b (or
    an upper bound; T when not given), which chooses the kernels.  Asynchronous on `stream`.  Returns (o, lse).
    """
    r = (_marshal_module or _native()).paged(0, q, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, o, lse,
                                             workspace, causal, scale, max_q, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_paged(_lib.attn_paged_fwd, torch.bfloat16, q, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale,
                          o, lse, workspace, causal, scale, max_q, stream)


def attn_paged_fwd_f16(q, k_pages, v_pages, page_table, start, kv_len, k_scale=None, v_scale=None, o=None, lse=None,
                       workspace=None, causal=True, scale=None, max_q=None, stream=None):
    """attn_paged_fwd_f16 on torch device tensors: as attn_paged_fwd, with fp16 q and o (and fp16 or e4m3 pages)."""
    r = (_marshal_module or _native()).paged(1, q, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, o, lse,
                                             workspace, causal, scale, max_q, stream)
    if r is not None:
        return _finish(r)
    import torch
    return _marshal_paged(_lib.attn_paged_fwd_f16, torch.float16, q, k_pages, v_pages, page_table, start, kv_len, k_scale,
                          v_scale, o, lse, workspace, causal, scale, max_q, stream)


def _marshal_paged(entry, dt, q, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, o, lse, workspace, causal, scale,
                   max_q, stream):
    import torch

    _check_rows(q, dt, 3, "q", q.device)
    T, H_q, D = q.shape
    kind, n_pages, H_kv, page_size, D_cache, B, width = _check_cache(dt, k_pages, v_pages, page_table, start, kv_len, k_scale,
                                                                     v_scale, q.device)
    if D != D_cache or H_kv < 1 or H_q % H_kv:
        raise ValueError("q's heads do not fit the cache's")
    need = attn_paged_fwd_workspace_bytes(T, B, H_q, H_kv, D)
    o = _allocate(lambda: torch.empty((T, H_q, D), dtype=dt, device=q.device), q.device, stream) if o is None else o
    if lse is None:
        lse = _allocate(lambda: torch.empty((T, H_q), dtype=torch.float32, device=q.device), q.device, stream)
    if workspace is None:
        workspace = _allocate(lambda: torch.empty((max(need, 16),), dtype=torch.uint8, device=q.device), q.device, stream,
                              returned=False)
    _check_array(o, dt, (T, H_q, D), "o", q.device)
    _check_array(lse, torch.float32, (T, H_q), "lse", q.device)
    _check_array(workspace, workspace.dtype, workspace.shape, "workspace", q.device)
    if scale is None:
        scale = 1.0 / float(D) ** 0.5
    if stream is None:
        stream = torch.cuda.current_stream(q.device)
    with torch.cuda.device(q.device):
        rc = entry(q.data_ptr(), _strides((q, 0), (q, 1)), o.data_ptr(), lse.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                   _address(k_scale), _address(v_scale), page_table.data_ptr(), start.data_ptr(), kv_len.data_ptr(), kind,
                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), T if max_q is None else min(int(max_q), _INT_MAX),
                   T, B, H_q, H_kv, D, n_pages, page_size, width, int(bool(causal)), float(scale), stream.cuda_stream)
    if rc != ATTN_OK:
        raise AttnError(rc)
    return o, lse
