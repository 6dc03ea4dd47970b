"""Python binding of the Rudder C-ABI library (``include/rudder.h``): argument marshalling only.

Every step of the quantized linear runs in the CUDA kernels behind the C ABI; torch is used for
device memory and streams.  There is no CPU fallback: if ``librudder.so`` is missing or cannot be
loaded, every call raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import numpy as np
import torch

_HERE = Path(__file__).resolve().parent
LIB_PATH = _HERE / "librudder.so"

# enums of rudder.h
OK, ERR_ARG, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(8)
W4A8_INT, W4A4_INT, W4A4_NVFP4 = 0, 1, 2
RANGE_PER_TOKEN, RANGE_STATIC = 0, 1
CACHE_BF16, CACHE_E4M3 = 0, 1
ROPE_HALF, ROPE_PAIRS = 0, 1
# second value of rudder_device_status after ERR_ARG: what a kernel found in the caller's device data
BAD_PAGE, BAD_LENGTH, BAD_POSITION, BAD_SLOT, NO_PAGES, NO_ROOM = range(911, 917)
SCHEMES = {"w4a8": W4A8_INT, "w4a4": W4A4_INT, "nvfp4": W4A4_NVFP4}

EXPORTED = [
    "rudder_pack_weights", "rudder_weight_free", "rudder_weight_info", "rudder_weight_export", "rudder_weight_import",
    "rudder_linear_workspace_bytes", "rudder_linear", "rudder_block_workspace_bytes", "rudder_block",
    "rudder_linear_static_max_workspace_bytes", "rudder_linear_static",
    "rudder_block_profile", "rudder_block_host_staging_bytes", "rudder_block_host",
    "rudder_quantize_activations", "rudder_linear_dump_acc", "rudder_device_status", "rudder_status_string",
    "rudder_gelu", "rudder_selftest_wait_timeout", "rudder_rmsnorm", "rudder_add",
    "rudder_block_dit", "rudder_block_dit_workspace_bytes", "rudder_gelu_quantize_activations",
    "rudder_page_tables", "rudder_qk_norm_rope", "rudder_attention_workspace_bytes", "rudder_attention_paged", "rudder_linear_a16",
    "rudder_block_cached_workspace_bytes", "rudder_block_cached",
]


class RudderError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class _ScaleTable(ctypes.Structure):
    _fields_ = [("gamma", ctypes.c_void_p), ("clip", ctypes.c_void_p), ("T", ctypes.c_int), ("S", ctypes.c_int),
                ("mode", ctypes.c_int)]


class _Segments(ctypes.Structure):
    _fields_ = [("seg_offsets", ctypes.POINTER(ctypes.c_int32)), ("seg_stream", ctypes.POINTER(ctypes.c_int32)),
                ("n_seg", ctypes.c_int)]


class _BlockGlue(ctypes.Structure):
    _fields_ = [("norm1_weight", ctypes.c_void_p), ("norm2_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("out", ctypes.c_void_p), ("ldout", ctypes.c_int64)]


class _BlockArgs(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p * 4), ("tab", ctypes.POINTER(_ScaleTable) * 4), ("bias", ctypes.c_void_p * 4),
                ("x", ctypes.c_void_p * 4), ("ldx", ctypes.c_int64 * 4), ("y", ctypes.c_void_p * 4),
                ("ldy", ctypes.c_int64 * 4)]


class _PagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("format", ctypes.c_int), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int),
                ("heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _PageTableArgs(ctypes.Structure):
    _fields_ = [("old_lens", ctypes.c_void_p), ("new_lens", ctypes.c_void_p), ("B", ctypes.c_int), ("page_size", ctypes.c_int),
                ("free_pages", ctypes.c_void_p), ("n_free", ctypes.c_int), ("page_table", ctypes.c_void_p), ("ld_table", ctypes.c_int64),
                ("max_pages", ctypes.c_int), ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("capacity", ctypes.c_int),
                ("starts", ctypes.c_void_p), ("used", ctypes.c_void_p)]


class _QkArgs(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("M", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("n_pos", ctypes.c_int), ("rot", ctypes.c_int), ("style", ctypes.c_int),
                ("positions", ctypes.c_void_p), ("Q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("K", ctypes.c_void_p), ("ldk", ctypes.c_int64),
                ("cache", ctypes.POINTER(_PagedCache)), ("slots", ctypes.c_void_p)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("Q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("M", ctypes.c_int), ("heads", ctypes.c_int), ("cache", ctypes.POINTER(_PagedCache)),
                ("page_table", ctypes.c_void_p), ("ld_table", ctypes.c_int64), ("max_pages", ctypes.c_int), ("kv_lens", ctypes.c_void_p),
                ("q_starts", ctypes.c_void_p), ("B", ctypes.c_int), ("max_q", ctypes.c_int), ("causal", ctypes.c_int), ("scale", ctypes.c_float),
                ("O", ctypes.c_void_p), ("ldo", ctypes.c_int64), ("lse", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library.  Raises if it has not been built (``python -m paper_2609_39056_b200.build``)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_39056_b200.build` "
                              "(there is no fallback path)")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        L.rudder_status_string.restype = ctypes.c_char_p
        L.rudder_status_string.argtypes = [i32]
        L.rudder_pack_weights.argtypes = [vp, vp, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
        L.rudder_weight_free.argtypes = [vp]
        L.rudder_weight_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                         ctypes.POINTER(i32), ctypes.POINTER(sz)]
        L.rudder_weight_export.argtypes = [vp, vp, vp, vp, vp, vp]
        L.rudder_weight_import.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
        L.rudder_linear_workspace_bytes.restype = sz
        L.rudder_linear_workspace_bytes.argtypes = [vp, i32]
        L.rudder_linear.argtypes = [vp, vp, i64, i32, ctypes.POINTER(_Segments), i32, ctypes.POINTER(_ScaleTable),
                                    vp, vp, i64, vp, sz, vp]
        L.rudder_linear_static_max_workspace_bytes.restype = sz
        L.rudder_linear_static_max_workspace_bytes.argtypes = []
        L.rudder_linear_static.argtypes = [vp, vp, i64, i32, ctypes.POINTER(_Segments), i32, ctypes.POINTER(_ScaleTable),
                                           vp, vp, i64, vp]
        L.rudder_block_workspace_bytes.restype = sz
        L.rudder_block_workspace_bytes.argtypes = [ctypes.POINTER(_BlockArgs), i32]
        L.rudder_block.argtypes = [ctypes.POINTER(_BlockArgs), i32, ctypes.POINTER(_Segments), i32, vp, sz, vp]
        L.rudder_block_profile.argtypes = [ctypes.POINTER(_BlockArgs), i32, ctypes.POINTER(_Segments), i32, vp, sz, vp,
                                           ctypes.POINTER(ctypes.c_float)]
        L.rudder_block_host_staging_bytes.restype = sz
        L.rudder_block_host_staging_bytes.argtypes = [ctypes.POINTER(_BlockArgs), i32]
        L.rudder_block_host.argtypes = [ctypes.POINTER(_BlockArgs), i32, ctypes.POINTER(_Segments), i32, vp, sz, vp, sz, vp]
        L.rudder_quantize_activations.argtypes = [vp, vp, i64, i32, ctypes.POINTER(_Segments), i32,
                                                  ctypes.POINTER(_ScaleTable), vp, vp, vp, vp]
        L.rudder_gelu_quantize_activations.argtypes = [vp, vp, i64, i32, ctypes.POINTER(_Segments), i32,
                                                       ctypes.POINTER(_ScaleTable), vp, vp, vp]
        L.rudder_linear_dump_acc.argtypes = [vp, vp, i64, i32, ctypes.POINTER(_Segments), i32,
                                             ctypes.POINTER(_ScaleTable), vp, vp, i64, vp, sz, vp,
                                             i32, i32, i32, i32, vp]
        L.rudder_device_status.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.rudder_gelu.argtypes = [vp, i64, i32, i32, vp, i64, vp]
        L.rudder_selftest_wait_timeout.argtypes = [ctypes.c_longlong, vp]
        L.rudder_rmsnorm.argtypes = [vp, i64, i32, i32, vp, ctypes.c_float, vp, i64, vp]
        L.rudder_add.argtypes = [vp, i64, vp, i64, i32, i32, vp, i64, vp]
        L.rudder_block_dit_workspace_bytes.restype = sz
        L.rudder_block_dit_workspace_bytes.argtypes = [ctypes.POINTER(_BlockArgs), i32]
        L.rudder_block_dit.argtypes = [ctypes.POINTER(_BlockArgs), ctypes.POINTER(_BlockGlue), i32, ctypes.POINTER(_Segments), i32, vp, sz, vp]
        L.rudder_page_tables.argtypes = [ctypes.POINTER(_PageTableArgs), vp]
        L.rudder_qk_norm_rope.argtypes = [ctypes.POINTER(_QkArgs), vp]
        L.rudder_attention_workspace_bytes.restype = sz
        L.rudder_attention_workspace_bytes.argtypes = [ctypes.POINTER(_AttentionArgs)]
        L.rudder_attention_paged.argtypes = [ctypes.POINTER(_AttentionArgs), vp, sz, vp]
        L.rudder_linear_a16.argtypes = [vp, vp, i64, i32, vp, vp, i64, vp]
        L.rudder_block_cached_workspace_bytes.restype = sz
        L.rudder_block_cached_workspace_bytes.argtypes = [ctypes.POINTER(_BlockArgs), ctypes.POINTER(_AttentionArgs), i32]
        L.rudder_block_cached.argtypes = [ctypes.POINTER(_BlockArgs), ctypes.POINTER(_BlockGlue), ctypes.POINTER(_QkArgs), ctypes.POINTER(_AttentionArgs),
                                          i32, ctypes.POINTER(_Segments), i32, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().rudder_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != OK:
        raise RudderError(status, what)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class Weight:
    """Owner of a ``rudder_weight*``; frees it when collected."""

    def __init__(self, handle, N, K, group, scheme, device_bytes):
        self.handle, self.N, self.K, self.group, self.scheme, self.device_bytes = handle, N, K, group, scheme, device_bytes

    def free(self):
        if self.handle:
            lib().rudder_weight_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


class ScaleTable:
    """Layer-step lookup table: gamma [T,S] fp32 (device), clip [T] fp32 (device) or None."""

    def __init__(self, gamma: torch.Tensor, clip: torch.Tensor | None = None, mode: int = RANGE_PER_TOKEN):
        assert gamma.dtype == torch.float32 and gamma.dim() == 2 and gamma.is_contiguous()
        assert clip is None or (clip.dtype == torch.float32 and clip.is_contiguous())
        self.gamma, self.clip, self.mode = gamma, clip, mode
        self.c = _ScaleTable(gamma.data_ptr(), clip.data_ptr() if clip is not None else None,
                             gamma.shape[0], gamma.shape[1], mode)


class Segments:
    """Row -> stream map: host arrays seg_offsets [n_seg+1], seg_stream [n_seg]."""

    def __init__(self, seg_offsets, seg_stream):
        self.off = np.ascontiguousarray(seg_offsets, dtype=np.int32)
        self.st = np.ascontiguousarray(seg_stream, dtype=np.int32)
        self.c = _Segments(self.off.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                           self.st.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), int(self.st.shape[0]))


def rudder_pack_weights(W: torch.Tensor, d: torch.Tensor | None, scheme: int, group: int, stream=None) -> Weight:
    assert W.is_cuda and W.dtype == torch.float32 and W.dim() == 2 and W.is_contiguous()
    assert d is None or (d.is_cuda and d.dtype == torch.float32 and d.is_contiguous())
    N, K = W.shape
    out = ctypes.c_void_p()
    _check(lib().rudder_pack_weights(_ptr(W), _ptr(d), N, K, int(scheme), int(group), _stream(stream),
                                     ctypes.byref(out)), "rudder_pack_weights")
    n, k, g, s, b = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(lib().rudder_weight_info(out, ctypes.byref(n), ctypes.byref(k), ctypes.byref(g), ctypes.byref(s),
                                    ctypes.byref(b)), "rudder_weight_info")
    return Weight(out, n.value, k.value, g.value, s.value, b.value)


def rudder_weight_export(w: Weight, stream=None):
    """Canonical view: codes uint8 [N,K/2], scales (int16 view of fp16 [N,K/G] | uint8 [N,K/16]), dinv, tensor_scale."""
    dev = torch.device("cuda", torch.cuda.current_device())
    codes = torch.empty((w.N, w.K // 2), dtype=torch.uint8, device=dev)
    if w.scheme == W4A4_NVFP4:
        scales = torch.empty((w.N, w.K // 16), dtype=torch.uint8, device=dev)
    else:
        scales = torch.empty((w.N, w.K // w.group), dtype=torch.float16, device=dev)
    dinv = torch.empty(w.K, dtype=torch.float32, device=dev)
    ts = torch.empty(1, dtype=torch.float32, device=dev)
    _check(lib().rudder_weight_export(w.handle, _ptr(codes), _ptr(scales), _ptr(dinv), _ptr(ts), _stream(stream)),
           "rudder_weight_export")
    return dict(codes=codes, scales=scales, dinv=dinv, tensor_scale=ts)


def rudder_weight_import(ex: dict, N: int, K: int, scheme: int, group: int, stream=None) -> Weight:
    """Packed weight from its canonical view (the dict rudder_weight_export returns)."""
    out = ctypes.c_void_p()
    _check(lib().rudder_weight_import(_ptr(ex["codes"]), _ptr(ex["scales"]), _ptr(ex["dinv"]), _ptr(ex.get("tensor_scale")),
                                      int(N), int(K), int(scheme), int(group), _stream(stream), ctypes.byref(out)),
           "rudder_weight_import")
    n, k, g, s, b = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(lib().rudder_weight_info(out, ctypes.byref(n), ctypes.byref(k), ctypes.byref(g), ctypes.byref(s),
                                    ctypes.byref(b)), "rudder_weight_info")
    return Weight(out, n.value, k.value, g.value, s.value, b.value)


def rudder_linear_workspace_bytes(w: Weight, M: int) -> int:
    return int(lib().rudder_linear_workspace_bytes(w.handle, int(M)))


def _workspace(nbytes, device, stream=None):
    """Scratch the binding allocates for the caller.  It is dropped when the call returns, while the kernels
    may still be running: torch's caching allocator only hands a freed block to later work of the stream it
    was allocated on, so the block is allocated under the stream the kernels are launched on."""
    if stream is None:
        return torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes + 256, dtype=torch.uint8, device=device)


def _aligned(ws: torch.Tensor):
    off = (-ws.data_ptr()) % 256
    return ctypes.c_void_p(ws.data_ptr() + off), ws.numel() - off


def rudder_linear(w: Weight, X: torch.Tensor, seg: Segments, step: int, tab: ScaleTable, bias=None, Y=None,
                  workspace=None, stream=None) -> torch.Tensor:
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M = X.shape[0]
    if Y is None:
        Y = torch.empty((M, w.N), dtype=torch.bfloat16, device=X.device)
    if workspace is None:
        workspace = _workspace(rudder_linear_workspace_bytes(w, M), X.device, stream)
    wp, wb = _aligned(workspace)
    _check(lib().rudder_linear(w.handle, _ptr(X), X.stride(0), M, ctypes.byref(seg.c), int(step), ctypes.byref(tab.c),
                               _ptr(bias), _ptr(Y), Y.stride(0), wp, wb, _stream(stream)), "rudder_linear")
    return Y


def rudder_linear_static_max_workspace_bytes() -> int:
    return int(lib().rudder_linear_static_max_workspace_bytes())


def rudder_linear_static(w: Weight, X: torch.Tensor, seg: Segments, step: int, tab: ScaleTable, bias=None, Y=None,
                         stream=None) -> torch.Tensor:
    """rudder_linear for callers that cannot allocate: the scratch between the two kernels is a fixed
    4 MiB array inside the library, so only inputs and the output are passed.  Raises
    RudderError(ERR_WORKSPACE) when the layer needs more scratch than the array holds.  Calls that may
    overlap on the GPU share the array and must be serialised by the caller."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M = X.shape[0]
    assert Y is not None, "the caller passes the output buffer: this entry point allocates nothing"
    _check(lib().rudder_linear_static(w.handle, _ptr(X), X.stride(0), M, ctypes.byref(seg.c), int(step),
                                      ctypes.byref(tab.c), _ptr(bias), _ptr(Y), Y.stride(0), _stream(stream)),
           "rudder_linear_static")
    return Y


def rudder_linear_dump_acc(w: Weight, X, seg, step, tab, bias=None, row0=0, rows=None, col0=0, cols=None, stream=None):
    """rudder_linear plus the INT32 group accumulators of a tile -> (Y, acc int32 [K/G, rows, cols])."""
    M = X.shape[0]
    rows = M - row0 if rows is None else rows
    cols = w.N - col0 if cols is None else cols
    Y = torch.empty((M, w.N), dtype=torch.bfloat16, device=X.device)
    acc = torch.full((w.K // w.group, rows, cols), -(2 ** 31), dtype=torch.int32, device=X.device)
    workspace = _workspace(rudder_linear_workspace_bytes(w, M), X.device, stream)
    wp, wb = _aligned(workspace)
    _check(lib().rudder_linear_dump_acc(w.handle, _ptr(X), X.stride(0), M, ctypes.byref(seg.c), int(step),
                                        ctypes.byref(tab.c), _ptr(bias), _ptr(Y), Y.stride(0), wp, wb, _stream(stream),
                                        int(row0), int(rows), int(col0), int(cols), _ptr(acc)),
           "rudder_linear_dump_acc")
    return Y, acc


def rudder_quantize_activations(w: Weight, X, seg, step, tab, stream=None):
    """First kernel alone -> (codes, block_scales | None, row_scale)."""
    M = X.shape[0]
    if w.scheme == W4A4_NVFP4:
        codes = torch.empty((M, w.K // 2), dtype=torch.uint8, device=X.device)
        sb = torch.empty((M, w.K // 16), dtype=torch.uint8, device=X.device)
    else:
        codes = torch.empty((M, w.K), dtype=torch.int8, device=X.device)
        sb = None
    r = torch.empty(M, dtype=torch.float32, device=X.device)
    _check(lib().rudder_quantize_activations(w.handle, _ptr(X), X.stride(0), M, ctypes.byref(seg.c), int(step),
                                             ctypes.byref(tab.c), _ptr(codes), _ptr(sb), _ptr(r), _stream(stream)),
           "rudder_quantize_activations")
    return codes, sb, r


class BlockArgs:
    """Arguments of rudder_block: 4 weights, tables, biases, replay inputs and outputs (QKV, O, up, down)."""

    def __init__(self, weights, tabs, biases, xs, ys):
        self.keep = (weights, tabs, biases, xs, ys)
        c = _BlockArgs()
        for l in range(4):
            c.w[l] = weights[l].handle
            c.tab[l] = ctypes.pointer(tabs[l].c)
            c.bias[l] = biases[l].data_ptr() if biases[l] is not None else None
            c.x[l] = xs[l].data_ptr() if xs[l] is not None else None        # None (l >= 1): chained to the previous output
            c.ldx[l] = xs[l].stride(0) if xs[l] is not None else 0
            c.y[l] = ys[l].data_ptr()
            c.ldy[l] = ys[l].stride(0)
        self.c = c


def rudder_gelu(X: torch.Tensor, Y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y = bf16(gelu(X)), elementwise, in the bit-defined form the chained block uses."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M, N = X.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    _check(lib().rudder_gelu(_ptr(X), X.stride(0), int(M), int(N), _ptr(Y), Y.stride(0), _stream(stream)), "rudder_gelu")
    return Y


def rudder_block_workspace_bytes(args: BlockArgs, M: int) -> int:
    return int(lib().rudder_block_workspace_bytes(ctypes.byref(args.c), int(M)))


def rudder_block(args: BlockArgs, M: int, seg: Segments, step: int, workspace: torch.Tensor, stream=None):
    wp, wb = _aligned(workspace)
    _check(lib().rudder_block(ctypes.byref(args.c), int(M), ctypes.byref(seg.c), int(step), wp, wb, _stream(stream)),
           "rudder_block")


def rudder_block_profile(args: BlockArgs, M: int, seg: Segments, step: int, workspace: torch.Tensor, stream=None):
    """rudder_block with an event between kernels -> 8 device times in ms (prologue, GEMM) x (QKV, O, up, down)."""
    wp, wb = _aligned(workspace)
    ms = (ctypes.c_float * 8)()
    _check(lib().rudder_block_profile(ctypes.byref(args.c), int(M), ctypes.byref(seg.c), int(step), wp, wb,
                                      _stream(stream), ms), "rudder_block_profile")
    return [float(v) for v in ms]


def rudder_block_host_staging_bytes(args: BlockArgs, M: int) -> int:
    return int(lib().rudder_block_host_staging_bytes(ctypes.byref(args.c), int(M)))


def rudder_block_host(args: BlockArgs, M: int, seg: Segments, step: int, staging: torch.Tensor,
                      workspace: torch.Tensor, stream=None):
    """rudder_block whose x / y tensors in ``args`` are (pinned) HOST tensors."""
    sp, sb = _aligned(staging)
    wp, wb = _aligned(workspace)
    _check(lib().rudder_block_host(ctypes.byref(args.c), int(M), ctypes.byref(seg.c), int(step), sp, sb, wp, wb,
                                   _stream(stream)), "rudder_block_host")


def rudder_device_status():
    """(last status, code of the wait that gave up); clears the device word.  Synchronises."""
    last, where = ctypes.c_int(), ctypes.c_int()
    _check(lib().rudder_device_status(ctypes.byref(last), ctypes.byref(where)), "rudder_device_status")
    return last.value, where.value


def rudder_selftest_wait_timeout(limit_cycles: int = 1_000_000, stream=None):
    """One warp waits `limit_cycles` SM clocks on a barrier nobody signals, gives up and records the time-out."""
    _check(lib().rudder_selftest_wait_timeout(int(limit_cycles), _stream(stream)), "rudder_selftest_wait_timeout")


def rudder_rmsnorm(X: torch.Tensor, weight: torch.Tensor, eps: float, Y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y = bf16((x / sqrt(mean(x^2) + eps)) * weight) per row, in the bit-defined form of the DiT block glue."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    assert weight.is_cuda and weight.dtype == torch.float32 and weight.is_contiguous() and weight.numel() == X.shape[1]
    M, N = X.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    _check(lib().rudder_rmsnorm(_ptr(X), X.stride(0), int(M), int(N), _ptr(weight), ctypes.c_float(eps), _ptr(Y), Y.stride(0),
                                _stream(stream)), "rudder_rmsnorm")
    return Y


def rudder_add(A: torch.Tensor, B: torch.Tensor, Y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y = bf16(A + B), elementwise (the residual addition of the DiT block glue)."""
    assert A.is_cuda and B.is_cuda and A.dtype == B.dtype == torch.bfloat16 and A.shape == B.shape and A.stride(1) == B.stride(1) == 1
    M, N = A.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    _check(lib().rudder_add(_ptr(A), A.stride(0), _ptr(B), B.stride(0), int(M), int(N), _ptr(Y), Y.stride(0), _stream(stream)), "rudder_add")
    return Y


def rudder_block_dit_workspace_bytes(args: BlockArgs, M: int) -> int:
    return int(lib().rudder_block_dit_workspace_bytes(ctypes.byref(args.c), int(M)))


def rudder_block_dit(args: BlockArgs, norm1_weight: torch.Tensor, norm2_weight: torch.Tensor, eps: float, out: torch.Tensor, M: int,
                     seg: Segments, step: int, workspace: torch.Tensor, stream=None):
    """One DiT block end to end from args.x[0]: norm -> QKV -> O (V third) -> + x -> norm -> up -> GELU -> down -> + h."""
    glue = _BlockGlue(norm1_weight.data_ptr(), norm2_weight.data_ptr(), float(eps), out.data_ptr(), out.stride(0))
    wp, wb = _aligned(workspace)
    _check(lib().rudder_block_dit(ctypes.byref(args.c), ctypes.byref(glue), int(M), ctypes.byref(seg.c), int(step), wp, wb,
                                  _stream(stream)), "rudder_block_dit")
    return out


def rudder_gelu_quantize_activations(w: Weight, X, seg, step, tab, stream=None):
    """The fused GELU + static-range prologue of a chained layer alone -> (codes int8 [M, K], row_scale)."""
    M = X.shape[0]
    codes = torch.empty((M, w.K), dtype=torch.int8, device=X.device)
    r = torch.empty(M, dtype=torch.float32, device=X.device)
    _check(lib().rudder_gelu_quantize_activations(w.handle, _ptr(X), X.stride(0), M, ctypes.byref(seg.c), int(step),
                                                  ctypes.byref(tab.c), _ptr(codes), _ptr(r), _stream(stream)),
           "rudder_gelu_quantize_activations")
    return codes, r


# ---- attention over a paged key-value cache, and what stands around it ------------------------------------------------------
# The argument objects hold the C structure and the tensors it points to: build one per set of buffers, call it every step.

def _on_one_device(*tensors) -> int:
    """The CUDA device index that all given tensors share (None entries are skipped)."""
    devs = {t.device for t in tensors if t is not None}
    if len(devs) != 1 or next(iter(devs)).type != "cuda":
        raise RudderError(ERR_ARG, f"tensors on one CUDA device expected, got {sorted(map(str, devs))}")
    return next(iter(devs)).index


def _launch_stream(device: int, stream):
    """Raw stream to launch on.  Like every call of the library, the buffers' device must be the current one."""
    if torch._C._cuda_getDevice() != device:
        raise RudderError(ERR_ARG, f"buffers are on device {device}, device {torch.cuda.current_device()} is current")
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(device)


def _int32(t, shape=None):
    assert t.dtype == torch.int32 and t.is_contiguous() and (shape is None or tuple(t.shape) == shape)


class PagedCache:
    """Keys and values of all requests: ``k`` and ``v`` [n_pages, heads, page_size, head_dim], bf16 or float8_e4m3fn, any strides with
    contiguous channels (a [n_pages, page_size, heads, head_dim] buffer is passed as ``.transpose(1, 2)``); ``k_scale`` / ``v_scale``
    fp32 [heads] for E4M3 (value = code x scale) or None."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
        assert k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.stride(3) == 1
        assert k.dtype in (torch.bfloat16, torch.float8_e4m3fn)
        for s in (k_scale, v_scale):
            assert s is None or (s.dtype == torch.float32 and s.is_contiguous() and s.numel() == k.shape[1])
        self.keep = (k, v, k_scale, v_scale)
        self.device = _on_one_device(k, v, k_scale, v_scale)
        self.n_pages, self.heads, self.page_size, self.head_dim = k.shape
        self.c = _PagedCache(k.data_ptr(), v.data_ptr(), CACHE_BF16 if k.dtype == torch.bfloat16 else CACHE_E4M3, self.n_pages, self.page_size,
                             self.heads, self.head_dim, k.stride(0), k.stride(1), k.stride(2),
                             k_scale.data_ptr() if k_scale is not None else None, v_scale.data_ptr() if v_scale is not None else None)


class PageTableArgs:
    """Arguments of rudder_page_tables: int32 device tensors except ``slots`` (int64); ``page_table`` [B, columns] is updated in place."""

    def __init__(self, old_lens, new_lens, free_pages, page_table, page_size: int, slots, positions, starts, used):
        B = old_lens.numel()
        _int32(old_lens, (B,)), _int32(new_lens, (B,)), _int32(free_pages), _int32(starts, (B + 1,)), _int32(used, (1,)), _int32(positions)
        assert page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.shape[0] == B and page_table.stride(1) == 1
        assert slots.dtype == torch.int64 and slots.is_contiguous() and slots.numel() == positions.numel()
        self.keep = (old_lens, new_lens, free_pages, page_table, slots, positions, starts, used)
        self.device = _on_one_device(*self.keep)
        self.c = _PageTableArgs(old_lens.data_ptr(), new_lens.data_ptr(), B, int(page_size), free_pages.data_ptr() if free_pages.numel() else None,
                                free_pages.numel(), page_table.data_ptr(), page_table.stride(0) if B > 1 else max(page_table.stride(0), page_table.shape[1]),
                                page_table.shape[1], slots.data_ptr(), positions.data_ptr(), positions.numel(), starts.data_ptr(), used.data_ptr())
        self.ref = ctypes.byref(self.c)


def rudder_page_tables(args: PageTableArgs, stream=None):
    """Page table, slots, positions and starts of a step from the requests' lengths, written into the tensors of ``args``."""
    _check(lib().rudder_page_tables(args.ref, _launch_stream(args.device, stream)), "rudder_page_tables")


def _rows(t: torch.Tensor) -> int:
    """Leading dimension of a [M, N] view with contiguous channels (one row has none of its own, whatever pitch its buffer has)."""
    assert t.dim() == 2 and t.stride(1) == 1
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 8) * 8


class QkArgs:
    """Arguments of rudder_qk_norm_rope.  ``X`` bf16 [M, (heads + 2 kv_heads) head_dim]; ``q_weight`` / ``k_weight`` fp32 [head_dim] or None;
    ``cos`` / ``sin`` fp32 [n_pos, rot / 2] or None (no rotation); ``positions`` int32 [M] (negative = row of padding); ``Q`` the output
    [M, heads head_dim]; keys to ``K`` [M, kv_heads head_dim], or keys and values to ``cache`` at ``slots`` int64 [M].
    For rudder_block_cached pass X = Q = None: the block supplies the rows."""

    def __init__(self, X, heads: int, kv_heads: int, head_dim: int, q_weight, k_weight, eps: float, cos, sin, style: int, positions, Q, K=None,
                 cache: PagedCache | None = None, slots=None):
        for w in (q_weight, k_weight):
            assert w is None or (w.dtype == torch.float32 and w.is_contiguous() and w.numel() == head_dim)
        assert (cos is None) == (sin is None)
        rot = 0
        if cos is not None:
            assert cos.dtype == sin.dtype == torch.float32 and cos.dim() == 2 and cos.shape == sin.shape and cos.is_contiguous() and sin.is_contiguous()
            rot = 2 * cos.shape[1]
        M = X.shape[0] if X is not None else (positions.numel() if positions is not None else slots.numel())
        if X is not None:
            assert X.dtype == Q.dtype == torch.bfloat16 and X.shape[1] == (heads + 2 * kv_heads) * head_dim and Q.shape == (M, heads * head_dim)
        assert K is None or (K.dtype == torch.bfloat16 and K.shape == (M, kv_heads * head_dim))
        if positions is not None:
            _int32(positions, (M,))
        assert slots is None or (slots.dtype == torch.int64 and slots.is_contiguous() and slots.numel() == M)
        self.keep = (X, q_weight, k_weight, cos, sin, positions, Q, K, slots)
        self.cache = cache
        self.device = _on_one_device(*self.keep, *(cache.keep if cache is not None else ()))
        p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
        self.c = _QkArgs(p(X), _rows(X) if X is not None else 0, M, int(heads), int(kv_heads), int(head_dim), p(q_weight), p(k_weight), float(eps),
                         p(cos), p(sin), cos.shape[0] if cos is not None else 0, rot, int(style), p(positions), p(Q), _rows(Q) if Q is not None else 0,
                         p(K), _rows(K) if K is not None else 0, ctypes.pointer(cache.c) if cache is not None else None, p(slots))
        self.ref = ctypes.byref(self.c)


def rudder_qk_norm_rope(args: QkArgs, stream=None):
    """Query / key norm per head, rotation and append to the cache, written into the tensors of ``args``."""
    _check(lib().rudder_qk_norm_rope(args.ref, _launch_stream(args.device, stream)), "rudder_qk_norm_rope")


class AttentionArgs:
    """Arguments of rudder_attention_paged.  ``Q`` and ``O`` bf16 [M, heads head_dim] (None for rudder_block_cached); ``page_table`` int32
    [B, columns]; ``kv_lens`` int32 [B]; ``q_starts`` int32 [B + 1] or None (rows b max_q .. of request b); ``lse`` fp32 [M, heads] or None."""

    def __init__(self, Q, heads: int, cache: PagedCache, page_table, kv_lens, scale: float, O, q_starts=None, max_q: int = 1, causal: bool = False, lse=None):
        B = kv_lens.numel()
        _int32(kv_lens, (B,))
        assert page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.shape[0] == B and page_table.stride(1) == 1
        if q_starts is not None:
            _int32(q_starts, (B + 1,))
        M = 0
        if Q is not None:
            M = Q.shape[0]
            assert Q.dtype == O.dtype == torch.bfloat16 and Q.shape == O.shape == (M, heads * cache.head_dim)
        assert lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and lse.dim() == 2 and lse.shape[1] == heads and (Q is None or lse.shape[0] == M))
        self.keep = (Q, page_table, kv_lens, O, q_starts, lse)
        self.cache = cache
        self.device = _on_one_device(*self.keep, *cache.keep)
        p = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
        self.c = _AttentionArgs(p(Q), _rows(Q) if Q is not None else 0, M, int(heads), ctypes.pointer(cache.c), page_table.data_ptr(),
                                page_table.stride(0) if B > 1 else max(page_table.stride(0), page_table.shape[1]), page_table.shape[1], kv_lens.data_ptr(),
                                p(q_starts), B, int(max_q), int(bool(causal)), float(scale), p(O), _rows(O) if O is not None else 0, p(lse))
        self.ref = ctypes.byref(self.c)


def rudder_attention_workspace_bytes(args: AttentionArgs) -> int:
    return int(lib().rudder_attention_workspace_bytes(args.ref))


def rudder_attention_paged(args: AttentionArgs, workspace: torch.Tensor | None = None, stream=None):
    """Attention of the new tokens over the cache, written into ``O`` (and ``lse``) of ``args``."""
    st = _launch_stream(args.device, stream)
    if workspace is None:
        workspace = _workspace(rudder_attention_workspace_bytes(args), args.keep[0].device, stream)
    p = workspace.data_ptr()
    off = -p % 256
    _check(lib().rudder_attention_paged(args.ref, p + off, workspace.numel() - off, st), "rudder_attention_paged")


def rudder_linear_a16(w: Weight, X: torch.Tensor, bias=None, Y=None, stream=None) -> torch.Tensor:
    """One to sixteen rows through a packed weight with 16-bit activations (no activation quantisation)."""
    M, K = X.shape
    ldx, one = X.stride()
    device = X.get_device()
    if Y is None:
        Y = torch.empty((M, w.N), dtype=torch.bfloat16, device=X.device)
    ldy, one_y = Y.stride()
    assert device >= 0 and X.dtype is torch.bfloat16 and K == w.K and one == 1
    assert Y.dtype is torch.bfloat16 and one_y == 1 and Y.shape == (M, w.N) and Y.get_device() == device
    b = None
    if bias is not None:
        assert bias.dtype is torch.float32 and bias.numel() == w.N and bias.is_contiguous() and bias.get_device() == device
        b = bias.data_ptr()
    if M == 1:                                       # one row has no leading dimension of its own
        ldx, ldy = K, w.N
    s = lib().rudder_linear_a16(w.handle, X.data_ptr(), ldx, M, b, Y.data_ptr(), ldy, _launch_stream(device, stream))
    if s:
        _check(s, "rudder_linear_a16")
    return Y


def rudder_block_cached_workspace_bytes(args: BlockArgs, attn: AttentionArgs, M: int) -> int:
    return int(lib().rudder_block_cached_workspace_bytes(ctypes.byref(args.c), attn.ref, int(M)))


def rudder_block_cached(args: BlockArgs, norm1_weight: torch.Tensor, norm2_weight: torch.Tensor, eps: float, out: torch.Tensor, qk: QkArgs, attn: AttentionArgs,
                        M: int, seg: Segments, step: int, workspace: torch.Tensor, stream=None):
    """rudder_block_dit with attention over the paged cache that ``qk`` and ``attn`` share in the place of its stand-in."""
    if qk.cache is not attn.cache:
        raise RudderError(ERR_ARG, "rudder_block_cached: qk and attn name different caches")
    qk.c.cache = attn.c.cache                        # one structure: the library compares the pointers
    glue = _BlockGlue(norm1_weight.data_ptr(), norm2_weight.data_ptr(), float(eps), out.data_ptr(), out.stride(0))
    wp, wb = _aligned(workspace)
    assert qk.c.M == M and (attn.keep[5] is None or attn.keep[5].shape[0] >= M)
    _check(lib().rudder_block_cached(ctypes.byref(args.c), ctypes.byref(glue), qk.ref, attn.ref, int(M), ctypes.byref(seg.c), int(step), wp, wb,
                                     _launch_stream(qk.device, stream)), "rudder_block_cached")
    return out
