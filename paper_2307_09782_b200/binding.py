"""Thin ctypes binding of ``libzqfp.so``: argument marshalling only.

Every function mirrors the C entry point of the same name in ``include/zqfp.h``.  Tensors are torch
CUDA tensors used purely as device memory; work is enqueued on torch's current stream.  There is no
CPU or PyTorch fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libzqfp.so")

SCALE_NONE, SCALE_M1, SCALE_M2 = 0, 1, 2
MODES = {"none": SCALE_NONE, "M1": SCALE_M1, "M2": SCALE_M2}
OUT_F32, OUT_BF16 = 0, 1
WEIGHTS_CAST, WEIGHTS_MX, WEIGHTS_MX_FP8, WEIGHTS_CAST_E5M2 = 0, 1, 2, 3
LAYOUTS = {"cast": WEIGHTS_CAST, "mx": WEIGHTS_MX, "mx_fp8": WEIGHTS_MX_FP8, "cast_e5m2": WEIGHTS_CAST_E5M2}

EXPORTS = [
    "zq_status_string", "zq_quantize_act_fp8", "zq_packed_weight_sizes", "zq_pack_weight_fp4",
    "zq_w4a8_linear_workspace_bytes", "zq_workspace_init", "zq_w4a8_linear",
    "zq_w4a8_linear_host_workspace_bytes", "zq_w4a8_linear_host", "zq_device_status", "zq_launch_count",
    "zq_w4a8_linear_noalloc_max_scratch_bytes", "zq_w4a8_linear_noalloc", "zq_w4a8_linear_noalloc_status", "zq_w4a8_linear_plan", "zq_selftest_bounded_wait", "zq_lorc_workspace_bytes", "zq_lorc_factors",
    "zq_w4a8_linear_fused_out", "zq_quantize_act_fp8_scaled", "zq_set_exclusive_device",
    "zq_quantize_fp8_block", "zq_quantize_weight_fp8_block", "zq_transpose_weight_fp8_block",
    "zq_fp8_block_workspace_bytes", "zq_fp8_block_linear", "zq_fp8_gated_linear", "zq_fp8_gated_linear_backward",
    "zq_fp8_weight_grad", "zq_fp8_gated_ffn_saved_bytes", "zq_fp8_gated_ffn_workspace_bytes", "zq_fp8_gated_ffn",
    "zq_fp8_gated_ffn_backward",
]
ACT_SILU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2
ACTIVATIONS = {"silu": ACT_SILU, "gelu_tanh": ACT_GELU_TANH, "relu": ACT_RELU}
PLAN_FIELDS = ("bm", "m_tiles", "n_tiles", "ctas", "stream", "persist", "splits", "kb_per_split", "base", "rem",
               "tail_pos0", "m_group", "partial_floats", "sms", "pair")


class ZqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib() -> C.CDLL:
    """Loads the library (building nothing: run ``__graft_entry__.build()`` first)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with paper_2307_09782_b200/build.py")
        L = C.CDLL(LIB_PATH)
        vp, i64, sz, ci = C.c_void_p, C.c_int64, C.c_size_t, C.c_int
        L.zq_status_string.restype = C.c_char_p
        L.zq_status_string.argtypes = [ci]
        L.zq_quantize_act_fp8.restype = ci
        L.zq_quantize_act_fp8.argtypes = [vp, i64, i64, i64, vp, vp, vp, ci, vp, vp]
        L.zq_packed_weight_sizes.restype = ci
        L.zq_packed_weight_sizes.argtypes = [i64, i64, ci, ci, ci, C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]
        L.zq_pack_weight_fp4.restype = ci
        L.zq_pack_weight_fp4.argtypes = [vp, i64, i64, ci, ci, ci, vp, vp, vp, vp]
        L.zq_w4a8_linear_workspace_bytes.restype = sz
        L.zq_w4a8_linear_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.zq_w4a8_linear_host_workspace_bytes.restype = sz
        L.zq_w4a8_linear_host_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.zq_workspace_init.restype = ci
        L.zq_workspace_init.argtypes = [vp, sz, vp]
        L.zq_w4a8_linear.restype = ci
        L.zq_w4a8_linear.argtypes = [vp, vp, vp, i64, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp, vp, vp, ci, vp, ci,
                                     i64, vp, sz, vp]
        L.zq_w4a8_linear_host.restype = ci
        L.zq_w4a8_linear_host.argtypes = [vp, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp, vp, ci, vp, vp, sz, vp]
        L.zq_w4a8_linear_plan.restype = ci
        L.zq_w4a8_linear_plan.argtypes = [i64, i64, i64, ci, ci, C.POINTER(i64)]
        L.zq_device_status.restype = ci
        L.zq_device_status.argtypes = [vp, C.POINTER(ci), vp]
        L.zq_launch_count.restype = i64
        L.zq_launch_count.argtypes = []
        L.zq_w4a8_linear_noalloc_max_scratch_bytes.restype = sz
        L.zq_w4a8_linear_noalloc_max_scratch_bytes.argtypes = []
        L.zq_w4a8_linear_noalloc.restype = ci
        L.zq_w4a8_linear_noalloc.argtypes = [vp, vp, i64, i64, i64, ci, ci, vp, vp, vp, vp, vp, ci, vp, ci, i64, vp]
        L.zq_w4a8_linear_noalloc_status.restype = ci
        L.zq_w4a8_linear_noalloc_status.argtypes = [C.POINTER(ci), vp]
        L.zq_selftest_bounded_wait.restype = ci
        L.zq_selftest_bounded_wait.argtypes = [vp, sz, C.c_uint32, vp]
        L.zq_lorc_workspace_bytes.restype = sz
        L.zq_lorc_workspace_bytes.argtypes = [i64, i64, ci]
        L.zq_lorc_factors.restype = ci
        L.zq_lorc_factors.argtypes = [vp, i64, i64, ci, ci, vp, vp, ci, vp, ci, vp, vp, vp, vp, sz, vp]
        L.zq_w4a8_linear_fused_out.restype = ci
        L.zq_w4a8_linear_fused_out.argtypes = L.zq_w4a8_linear.argtypes + [ci, vp]
        L.zq_quantize_act_fp8_scaled.restype = ci
        L.zq_quantize_act_fp8_scaled.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, ci, vp, vp]
        L.zq_set_exclusive_device.restype = ci
        L.zq_set_exclusive_device.argtypes = [ci]
        L.zq_quantize_fp8_block.restype = ci
        L.zq_quantize_fp8_block.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp]
        L.zq_quantize_weight_fp8_block.restype = ci
        L.zq_quantize_weight_fp8_block.argtypes = [vp, i64, i64, ci, vp, vp, vp]
        L.zq_transpose_weight_fp8_block.restype = ci
        L.zq_transpose_weight_fp8_block.argtypes = [vp, vp, i64, i64, vp, vp, vp]
        L.zq_fp8_block_workspace_bytes.restype = sz
        L.zq_fp8_block_workspace_bytes.argtypes = [i64, i64]
        L.zq_fp8_block_linear.restype = ci
        L.zq_fp8_block_linear.argtypes = [vp, vp, vp, i64, ci, ci, i64, i64, i64, vp, vp, vp, ci, i64, vp, sz, vp]
        L.zq_fp8_gated_linear.restype = ci
        L.zq_fp8_gated_linear.argtypes = [vp, vp, vp, i64, ci, i64, i64, i64, vp, vp, ci, vp, i64, vp, vp, vp, vp, vp, sz,
                                          vp]
        L.zq_fp8_gated_linear_backward.restype = ci
        L.zq_fp8_gated_linear_backward.argtypes = [vp, vp, vp, i64, ci, i64, i64, i64, vp, vp, ci, vp, vp, vp, vp, vp, vp,
                                                   sz, vp]
        L.zq_fp8_gated_ffn_saved_bytes.restype = sz
        L.zq_fp8_gated_ffn_saved_bytes.argtypes = [i64, i64, i64]
        L.zq_fp8_gated_ffn_workspace_bytes.restype = sz
        L.zq_fp8_gated_ffn_workspace_bytes.argtypes = [i64, i64, i64, i64, ci]
        L.zq_fp8_gated_ffn.restype = ci
        L.zq_fp8_gated_ffn.argtypes = [vp, i64, ci, i64, i64, i64, i64, vp, vp, vp, vp, ci, vp, ci, i64, vp, vp, sz, vp]
        L.zq_fp8_gated_ffn_backward.restype = ci
        L.zq_fp8_gated_ffn_backward.argtypes = [vp, i64, ci, i64, i64, i64, i64, vp, vp, vp, vp, vp, ci, vp, vp, vp, ci, vp,
                                                sz, vp]
        L.zq_fp8_weight_grad.restype = ci
        L.zq_fp8_weight_grad.argtypes = [vp, i64, i64, ci, vp, vp, i64, i64, i64, vp, ci, vp, sz, vp]
        _lib = L
    return _lib


def set_exclusive_device(on: bool) -> bool:
    """``zq_set_exclusive_device``: promise that nothing else runs on the device; returns the previous setting."""
    return bool(lib().zq_set_exclusive_device(1 if on else 0))


def status_string(status: int) -> str:
    return lib().zq_status_string(int(status)).decode()


def launch_count() -> int:
    return int(lib().zq_launch_count())


def _mode(mode) -> int:
    return MODES[mode] if isinstance(mode, str) else int(mode)


def _layout(layout) -> int:
    return LAYOUTS[layout] if isinstance(layout, str) else int(layout)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    """The current stream's handle (torch.cuda.current_stream().cuda_stream, without building a Stream object: 3 us)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _capturing() -> bool:
    """Whether calls on the current stream are being captured into a CUDA graph."""
    return torch._C._cuda_isCurrentStreamCapturing()


def _check(status: int, where: str):
    if status != 0:
        raise ZqError(status, where)


def _out_type(dtype) -> int:
    """The library's name for a result type.  Any other type would be written as bf16: wrong bits, or beyond its end."""
    if dtype is torch.bfloat16:
        return OUT_BF16
    if dtype is torch.float32:
        return OUT_F32
    raise ValueError(f"out_dtype: torch.float32 or torch.bfloat16 is needed, got {dtype}")


def packed_weight_sizes(N: int, K: int, group: int, mode, layout=WEIGHTS_CAST):
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(lib().zq_packed_weight_sizes(N, K, group, _mode(mode), _layout(layout), C.byref(a), C.byref(b),
                                        C.byref(c)),
           "zq_packed_weight_sizes")
    return a.value, b.value, c.value


def quantize_act_fp8(x: torch.Tensor, V: Optional[torch.Tensor] = None, absmax: Optional[torch.Tensor] = None):
    """x: bf16 [M, K] (row stride allowed).  Returns (q uint8 [M,K], sx float32 [M], t float32 [M,r] | None).
    With ``absmax`` (float32 [M], the rows' exact absolute maxima): ``zq_quantize_act_fp8_scaled``, one pass."""
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    M, K = x.shape
    q = torch.empty((M, K), dtype=torch.uint8, device=x.device)
    sx = torch.empty((M,), dtype=torch.float32, device=x.device)
    r, t = 0, None
    if V is not None:
        assert V.dtype == torch.float16 and V.is_contiguous() and V.shape[1] == K
        r = V.shape[0]
        t = torch.empty((M, r), dtype=torch.float32, device=x.device)
    ldx = x.stride(0) if M > 1 else K
    if absmax is not None:
        assert absmax.dtype == torch.float32 and absmax.is_contiguous() and absmax.shape == (M,)
        _check(lib().zq_quantize_act_fp8_scaled(_ptr(x), M, K, ldx, _ptr(absmax), _ptr(q), _ptr(sx), _ptr(V), r,
                                                _ptr(t), _stream()), "zq_quantize_act_fp8_scaled")
        return q, sx, t
    _check(lib().zq_quantize_act_fp8(_ptr(x), M, K, ldx, _ptr(q), _ptr(sx), _ptr(V), r, _ptr(t), _stream()),
           "zq_quantize_act_fp8")
    return q, sx, t


@dataclass
class PackedWeight:
    """Device buffers written by ``zq_pack_weight_fp4`` plus the shape they were packed for."""
    codes: torch.Tensor               # uint8, tiled layout (see include/zqfp.h)
    shift: Optional[torch.Tensor]     # uint8 [N, G] (M1, M2) or None
    scale: torch.Tensor               # float32 [N] (M1, M2) or [N, G] (none)
    N: int
    K: int
    group: int
    mode: int
    layout: int = WEIGHTS_CAST

    def clone(self) -> "PackedWeight":
        return PackedWeight(self.codes.clone(), None if self.shift is None else self.shift.clone(),
                            self.scale.clone(), self.N, self.K, self.group, self.mode, self.layout)


def pack_weight_fp4(W: torch.Tensor, group: int, mode, layout=WEIGHTS_CAST) -> PackedWeight:
    """W: float32 [N, K] contiguous.  ``layout``: "cast" (the kernel casts FP4 to FP8) or "mx" (the tensor core does)."""
    assert W.dtype == torch.float32 and W.is_contiguous() and W.dim() == 2
    N, K = W.shape
    mode = _mode(mode)
    layout = _layout(layout)
    cb, sb, fb = packed_weight_sizes(N, K, group, mode, layout)
    G = K // group
    codes = torch.empty((cb,), dtype=torch.uint8, device=W.device)
    shift = None if mode == SCALE_NONE else torch.empty((N, G), dtype=torch.uint8, device=W.device)
    scale = torch.empty((N, G) if mode == SCALE_NONE else (N,), dtype=torch.float32, device=W.device)
    assert scale.numel() * 4 == fb and (shift is None or shift.numel() == sb)
    _check(lib().zq_pack_weight_fp4(_ptr(W), N, K, group, mode, layout, _ptr(codes), _ptr(shift), _ptr(scale),
                                    _stream()), "zq_pack_weight_fp4")
    return PackedWeight(codes, shift, scale, N, K, group, mode, layout)


def linear_plan(M: int, N: int, K: int, mode, layout=WEIGHTS_CAST) -> dict:
    """The launch plan ``zq_w4a8_linear`` would use (host only, nothing is launched)."""
    out = (C.c_int64 * len(PLAN_FIELDS))()
    _check(lib().zq_w4a8_linear_plan(M, N, K, _mode(mode), _layout(layout), out), "zq_w4a8_linear_plan")
    return dict(zip(PLAN_FIELDS, [int(v) for v in out]))


def linear_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    return int(lib().zq_w4a8_linear_workspace_bytes(M, N, K, r))


def linear_host_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    return int(lib().zq_w4a8_linear_host_workspace_bytes(M, N, K, r))


def make_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Allocates (through torch) and zero-initializes a workspace of ``nbytes``."""
    ws = torch.empty((max(int(nbytes), 1),), dtype=torch.uint8, device=device)
    _check(lib().zq_workspace_init(_ptr(ws), ws.numel(), _stream()), "zq_workspace_init")
    return ws


def w4a8_linear(w: PackedWeight, *, q=None, sx=None, t=None, x=None, U=None, V=None,
                out_dtype=torch.float32, workspace: Optional[torch.Tensor] = None, y=None, relu=False,
                y_absmax: Optional[torch.Tensor] = None):
    """y [M, N] = the quantized linear layer; activations either (q, sx[, t]) or raw bf16 ``x`` (then V when U).
    ``relu`` / ``y_absmax`` (float32 [M], written): ``zq_w4a8_linear_fused_out``."""
    codes, shift, scale, group, mode, N, K = w.codes, w.shift, w.scale, w.group, w.mode, w.N, w.K
    if x is not None:
        M, ldx = x.shape[0], (x.stride(0) if x.shape[0] > 1 else K)
    else:
        M, ldx = q.shape[0], K
    r = 0 if U is None else U.shape[1]
    if workspace is None:
        workspace = make_workspace(linear_workspace_bytes(M, N, K, r), codes.device)
    ydt = _out_type(out_dtype if y is None else y.dtype)
    if y is None:
        y = torch.empty((M, N), dtype=out_dtype, device=codes.device)
    ldy = y.stride(0) if M > 1 else N
    if relu or y_absmax is not None:
        assert y_absmax is None or (y_absmax.dtype == torch.float32 and y_absmax.is_contiguous() and
                                    y_absmax.shape == (M,))
        _check(lib().zq_w4a8_linear_fused_out(_ptr(q), _ptr(sx), _ptr(x), ldx, M, N, K, group, _mode(mode), w.layout,
                                              _ptr(codes), _ptr(shift), _ptr(scale), _ptr(U), _ptr(V), _ptr(t), r,
                                              _ptr(y), ydt, ldy, _ptr(workspace), workspace.numel(), _stream(),
                                              1 if relu else 0, _ptr(y_absmax)), "zq_w4a8_linear_fused_out")
        return y
    _check(lib().zq_w4a8_linear(_ptr(q), _ptr(sx), _ptr(x), ldx, M, N, K, group, _mode(mode), w.layout, _ptr(codes),
                                _ptr(shift), _ptr(scale), _ptr(U), _ptr(V), _ptr(t), r, _ptr(y), ydt, ldy,
                                _ptr(workspace), workspace.numel(), _stream()), "zq_w4a8_linear")
    return y


def w4a8_linear_noalloc(w: PackedWeight, *, q, sx, t=None, U=None, y=None, out_dtype=torch.float32):
    """``zq_w4a8_linear_noalloc``: same result as :func:`w4a8_linear` on pre-quantized activations, for
    callers that cannot allocate a workspace; the scratch is a fixed array inside the library."""
    codes, shift, scale, group, mode, N, K = w.codes, w.shift, w.scale, w.group, w.mode, w.N, w.K
    assert w.layout == WEIGHTS_CAST, "zq_w4a8_linear_noalloc takes weights in the cast layout"
    M = q.shape[0]
    r = 0 if U is None else U.shape[1]
    ydt = _out_type(out_dtype if y is None else y.dtype)
    if y is None:
        y = torch.empty((M, N), dtype=out_dtype, device=codes.device)
    ldy = y.stride(0) if M > 1 else N
    _check(lib().zq_w4a8_linear_noalloc(_ptr(q), _ptr(sx), M, N, K, group, _mode(mode), _ptr(codes), _ptr(shift),
                                        _ptr(scale), _ptr(U), _ptr(t), r, _ptr(y), ydt, ldy, _stream()),
           "zq_w4a8_linear_noalloc")
    return y


def lorc_factors(W: torch.Tensor, w: "PackedWeight", r: int, omega: torch.Tensor, iters: int = 2):
    """LoRC factors of W - dequant(w): returns (U^ fp16 [N,r], V^ fp16 [r,K], sigma2 float32 [r])."""
    assert W.dtype == torch.float32 and W.is_contiguous() and omega.dtype == torch.float32 and omega.is_contiguous()
    N, K = W.shape
    assert omega.shape == (K, r + 8)
    U = torch.empty((N, r), dtype=torch.float16, device=W.device)
    V = torch.empty((r, K), dtype=torch.float16, device=W.device)
    s2 = torch.empty((r,), dtype=torch.float32, device=W.device)
    ws = torch.empty((max(int(lib().zq_lorc_workspace_bytes(N, K, r)), 1),), dtype=torch.uint8, device=W.device)
    _check(lib().zq_lorc_factors(_ptr(W), N, K, w.group, _mode(w.mode), _ptr(w.shift), _ptr(w.scale), r, _ptr(omega),
                                 iters, _ptr(U), _ptr(V), _ptr(s2), _ptr(ws), ws.numel(), _stream()), "zq_lorc_factors")
    return U, V, s2


def selftest_bounded_wait(workspace: torch.Tensor, limit_us: int = 1000):
    """Launches the kernel whose bounded wait is meant to run out; read the outcome with device_status()."""
    _check(lib().zq_selftest_bounded_wait(_ptr(workspace), workspace.numel(), int(limit_us), _stream()),
           "zq_selftest_bounded_wait")


def noalloc_status():
    """Synchronizes the current stream; returns (status, detail) of the fixed scratch array and clears them."""
    d = C.c_int(0)
    st = lib().zq_w4a8_linear_noalloc_status(C.byref(d), _stream())
    return int(st), int(d.value)


def w4a8_linear_host(x_host: torch.Tensor, y_host: torch.Tensor, w: PackedWeight, *, U=None, V=None,
                     workspace: torch.Tensor):
    """Host-buffer variant: x_host bf16 [M,K] and y_host float32 [M,N] are CPU (pinned) tensors; synchronous."""
    assert not x_host.is_cuda and not y_host.is_cuda and x_host.is_contiguous() and y_host.is_contiguous()
    codes, shift, scale, group, mode, N = w.codes, w.shift, w.scale, w.group, w.mode, w.N
    M, K = x_host.shape
    assert K == w.K
    r = 0 if U is None else U.shape[1]
    _check(lib().zq_w4a8_linear_host(_ptr(x_host), M, N, K, group, _mode(mode), w.layout, _ptr(codes), _ptr(shift),
                                     _ptr(scale), _ptr(U), _ptr(V), r, _ptr(y_host), _ptr(workspace),
                                     workspace.numel(), _stream()), "zq_w4a8_linear_host")
    return y_host


def device_status(workspace: torch.Tensor):
    """Synchronizes the current stream; returns (status, detail)."""
    d = C.c_int(0)
    st = lib().zq_device_status(_ptr(workspace), C.byref(d), _stream())
    return int(st), int(d.value)


# ---- FP8 with block scales --------------------------------------------------------------------------

def _version(t: torch.Tensor) -> int:
    """A number that changes when torch writes to a tensor (inference tensors have none)."""
    return -1 if t.is_inference() else t._version


class _ScalesPow2:
    """``pow2``: whether all scales are powers of two, as far as it is known: of these scales, as they were written last.  (Writes
    that torch does not count, through ``.data``, by a kernel of one's own or to an inference tensor, are the caller's to
    tell: set ``pow2`` anew.)"""

    def _known_pow2(self) -> Optional[bool]:
        scale, version, value = self._pow2
        return value if scale is self.scale and version == _version(scale) else None

    def _set_pow2(self, value: Optional[bool]):
        self._pow2 = self.scale, _version(self.scale), value

    def __getstate__(self):  # (a copied tensor counts its writes anew)
        return {**self.__dict__, "_pow2": self._known_pow2()}

    def __setstate__(self, state):
        known = state.pop("_pow2")
        self.__dict__.update(state)
        self._set_pow2(known)


@dataclass
class Fp8Block(_ScalesPow2):
    """Activations as E4M3 codes with one scale per row and 128 features (``zq_quantize_fp8_block``)."""
    codes: torch.Tensor   # uint8 [M, K] (or [parts, M, K])
    scale: torch.Tensor   # float32 [ceil(K / 128), M] (or [parts, ...]): the row index is innermost
    pow2: bool = False    # the scales are known to be powers of two (mode "M1")

    def values(self) -> torch.Tensor:
        """The FP32 values the codes stand for (a convenience for inspection, not a hot path)."""
        K = self.codes.shape[-1]
        s = self.scale.transpose(-1, -2).repeat_interleave(128, -1)[..., :K]
        return self.codes.view(torch.float8_e4m3fn).float() * s


Fp8Block.pow2 = property(lambda self: bool(self._known_pow2()), _ScalesPow2._set_pow2)


@dataclass
class Fp8Weight(_ScalesPow2):
    """Weights as E4M3 codes with one scale per 128 x 128 block (``zq_quantize_weight_fp8_block``); ``parts`` = 2 for the
    stacked gate and up projections."""
    codes: torch.Tensor   # uint8 [N, K] or [parts, N, K]
    scale: torch.Tensor   # float32 [ceil(N / 128), ceil(K / 128)] or [parts, ...]
    N: int
    K: int
    parts: int = 1
    pow2: Optional[bool] = None   # whether all scales are powers of two; None: looked up when it is first needed

    def __post_init__(self):
        lead = (self.parts,) if self.parts > 1 else ()
        nb, kb = (self.N + 127) // 128, (self.K + 127) // 128
        if tuple(self.codes.shape) != (*lead, self.N, self.K) or tuple(self.scale.shape) != (*lead, nb, kb):
            raise ValueError(f"codes {tuple(self.codes.shape)} / scales {tuple(self.scale.shape)} do not belong to "
                             f"{self.parts} x [{self.N}, {self.K}]")
        _expect(self.codes, torch.uint8, "codes")
        _expect(self.scale, torch.float32, "scale")

    def _look_up_pow2(self) -> bool:
        value = self._known_pow2()
        if value is None:
            if not self.scale.is_cuda or _capturing():  # (a capture cannot wait for the answer)
                return False
            bits = self.scale.view(torch.int32)  # positive, finite, no zero, a mantissa of zero
            self.pow2 = value = bool((((bits & 0x7FFFFF) == 0) & (bits > 0) & (bits < 0x7F800000)).all())
        return value

    def values(self) -> torch.Tensor:
        s = self.scale.repeat_interleave(128, -1)[..., :self.K].repeat_interleave(128, -2)[..., :self.N, :]
        return self.codes.view(torch.float8_e4m3fn).float() * s


Fp8Weight.pow2 = property(Fp8Weight._look_up_pow2, _ScalesPow2._set_pow2)


def _expect(t: torch.Tensor, dtype, name: str):
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor is needed, got {t.dtype}, strides {t.stride()}")


def _on_gpu(*tensors: torch.Tensor):
    """The library takes device pointers and launches on the current device: a tensor in host memory, or on another device,
    must not get that far."""
    here = None
    for t in tensors:
        d = t.get_device()  # -1: host memory
        if d != here:
            if d < 0:
                raise ValueError(f"a CUDA tensor is needed, got one of {tuple(t.shape)} on {t.device}")
            here = torch._C._cuda_getDevice()
            if d != here:
                raise ValueError(f"a tensor of {tuple(t.shape)} is on cuda:{d}, the current device is cuda:{here}: call under "
                                 f"torch.cuda.device({d}), with all tensors there")


def _rows(x: torch.Tensor, name: str):
    """(row stride, rows, columns) of a bf16 matrix whose rows are contiguous."""
    if x.dtype is torch.bfloat16 and x.dim() == 2:
        M, K = x.shape
        ld, step = x.stride()
        if step == 1 or K <= 1:
            return ld if M > 1 else (K + 7) // 8 * 8, M, K
    raise ValueError(f"{name}: a bf16 matrix with contiguous rows is needed, got {x.dtype} {tuple(x.shape)}, "
                     f"strides {x.stride()}")


def fp8_block_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    """Workspace for :func:`fp8_block_linear` and the gated layers on M rows of K features (N does not matter)."""
    return int(lib().zq_fp8_block_workspace_bytes(M, K))


def _blocks(n: int) -> int:
    return (n + 127) // 128


def quantize_fp8_block(x: torch.Tensor, mode="none") -> Fp8Block:
    """x: bf16 [M, K] (row stride allowed); ``mode`` "none" (FP32 scales) or "M1" (powers of two)."""
    ldx, M, K = _rows(x, "x")
    _on_gpu(x)
    q = x.new_empty((M, K), dtype=torch.uint8)
    s = x.new_empty(((K + 127) // 128, M), dtype=torch.float32)
    _check(lib().zq_quantize_fp8_block(_ptr(x), M, K, ldx, _mode(mode), _ptr(q), _ptr(s), _stream()),
           "zq_quantize_fp8_block")
    return Fp8Block(q, s, _mode(mode) == SCALE_M1)


def quantize_weight_fp8_block(W: torch.Tensor, mode="none") -> Fp8Weight:
    """W: float32 [N, K] or [parts, N, K], contiguous."""
    _expect(W, torch.float32, "W")
    _on_gpu(W)
    parts = W.shape[0] if W.dim() == 3 else 1
    N, K = W.shape[-2:]
    lead = W.shape[:-2] if parts > 1 else ()
    q = torch.empty((*lead, N, K), dtype=torch.uint8, device=W.device)
    s = torch.empty((*lead, _blocks(N), _blocks(K)), dtype=torch.float32, device=W.device)
    for i in range(parts):
        Wi, qi, si = (W.view(parts, N, K)[i], q.view(parts, N, K)[i], s.view(parts, _blocks(N), _blocks(K))[i])
        _check(lib().zq_quantize_weight_fp8_block(_ptr(Wi), N, K, _mode(mode), _ptr(qi), _ptr(si), _stream()),
               "zq_quantize_weight_fp8_block")
    return Fp8Weight(q, s, N, K, parts, _mode(mode) == SCALE_M1)


def transpose_fp8_weight(w: Fp8Weight) -> Fp8Weight:
    """The transposed weight (of each part): [N, K] -> [K, N]."""
    _on_gpu(w.codes, w.scale)
    lead = (w.parts,) if w.parts > 1 else ()
    nb, kb = _blocks(w.N), _blocks(w.K)
    q = torch.empty((*lead, w.K, w.N), dtype=torch.uint8, device=w.codes.device)
    s = torch.empty((*lead, kb, nb), dtype=torch.float32, device=w.codes.device)
    for i in range(w.parts):
        _check(lib().zq_transpose_weight_fp8_block(
            _ptr(w.codes.view(w.parts, w.N, w.K)[i]), _ptr(w.scale.view(w.parts, nb, kb)[i]), w.N, w.K,
            _ptr(q.view(w.parts, w.K, w.N)[i]), _ptr(s.view(w.parts, kb, nb)[i]), _stream()),
            "zq_transpose_weight_fp8_block")
    return Fp8Weight(q, s, w.K, w.N, w.parts, w._known_pow2())


def _activations(x, q, K: int, parts: int, *others: torch.Tensor):
    """(codes, scales, x, ldx, M) of an operand given raw (``x``) or quantized (``q``); it and the ``others`` are on the GPU."""
    if (x is None) == (q is None):
        raise ValueError("give the activations either raw (x) or quantized (q)")
    if x is not None:
        ldx, M, features = _rows(x, "x")
        if features != K:
            raise ValueError(f"x has {features} features, the weight {K}")
        _on_gpu(x, *others)
        return None, None, x, ldx, M
    _expect(q.codes, torch.uint8, "q.codes")
    _expect(q.scale, torch.float32, "q.scale")
    M = q.codes.shape[-2]
    lead = (parts,) if parts > 1 else ()
    if tuple(q.codes.shape) != (*lead, M, K) or tuple(q.scale.shape) != (*lead, _blocks(K), M):
        raise ValueError(f"codes {tuple(q.codes.shape)} / scales {tuple(q.scale.shape)} do not fit {parts} x [M, {K}]")
    _on_gpu(q.codes, q.scale, *others)
    return q.codes, q.scale, None, K, M


SCALES_POW2 = 16


def _scales(mode, w: Fp8Weight, q: Optional[Fp8Block]) -> int:
    """The scale rule, with the promise of ``ZQ_SCALES_POW2`` where every scale the call is given is a power of two."""
    m = _mode(mode)
    return m | SCALES_POW2 if (m == SCALE_M1 if q is None else q.pow2) and w.pow2 else m


def _ffn_scales(mode, gate_up: Fp8Weight, down: Fp8Weight) -> int:
    m = _scales(mode, gate_up, None)
    return m if m & SCALES_POW2 and down.pow2 else _mode(mode)


class KeptWorkspaces(threading.local):
    """Workspaces that outlast a call, each thread's own: the library is called without the interpreter's lock, so the kernels of
    two threads' calls can mix on a stream that they share.  Copies and pickles start empty."""

    def __init__(self):
        self.of = {}

    def __reduce__(self):
        return KeptWorkspaces, ()


_fp8_workspaces = KeptWorkspaces()
_fp8_head = 0


def _fp8_workspace_need(M: int, K: int) -> int:
    """``zq_fp8_block_workspace_bytes`` without a call into the library: a head, the codes, the scales, each rounded up to 256."""
    global _fp8_head
    if _fp8_head == 0:
        _fp8_head = int(lib().zq_fp8_block_workspace_bytes(0, 16))
    return _fp8_head + (M * K + 255) // 256 * 256 + (4 * M * _blocks(K) + 255) // 256 * 256


def _fp8_workspace(workspace, M: int, K: int, device):
    """The caller's workspace, or one that is kept per thread, device and stream and grown on demand.  A call that is captured into a
    CUDA graph gets one of its own, in the graph's memory: a graph lasts longer than a kept one, which is given back when it
    has to grow, and may be replayed on any stream."""
    if workspace is not None:
        _expect(workspace, torch.uint8, "workspace")
        _on_gpu(workspace)
        return workspace
    need = _fp8_workspace_need(M, K)
    if _capturing():
        return make_workspace(need, device)
    key = (device.index, _stream())
    kept = _fp8_workspaces.of
    ws = kept.get(key)
    if ws is None or ws.numel() < need:
        ws = kept[key] = make_workspace(need, device)
    return ws


def fp8_block_linear(w: Fp8Weight, *, x=None, q: Optional[Fp8Block] = None, mode="none", out_dtype=torch.float32, y=None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [M, N] = the linear layer; activations raw (bf16 ``x``, quantized with ``mode``) or quantized (``q``).  With
    ``w.parts`` = 2 the sum over two pairs of operands (``q`` then holds two as well)."""
    ydt = _out_type(out_dtype if y is None else y.dtype)
    codes, scale, x, ldx, M = _activations(x, q, w.K, w.parts, w.codes, w.scale)
    if y is None:
        y = w.scale.new_empty((M, w.N), dtype=out_dtype)
    else:
        if y.shape != (M, w.N) or (w.N > 1 and y.stride(1) != 1):
            raise ValueError(f"y: a [{M}, {w.N}] matrix with contiguous rows is needed")
        _on_gpu(y)
    workspace = _fp8_workspace(workspace, M, w.K, w.codes.device)
    _check(lib().zq_fp8_block_linear(_ptr(codes), _ptr(scale), _ptr(x), ldx, _scales(mode, w, q), w.parts, M, w.N, w.K,
                                     _ptr(w.codes), _ptr(w.scale), _ptr(y), ydt, y.stride(0) if M > 1 else w.N,
                                     _ptr(workspace), workspace.numel(), _stream()), "zq_fp8_block_linear")
    return y


def _act(act) -> int:
    return ACTIVATIONS[act] if isinstance(act, str) else int(act)


def fp8_gated_linear(w: Fp8Weight, *, x=None, q: Optional[Fp8Block] = None, act="silu", mode="none", bf16=True,
                     quantized=False, checkpoint=False, workspace: Optional[torch.Tensor] = None):
    """h = act(x Wg^T) * (x Wu^T) with ``w`` the stacked (gate, up) weights.  Returns (h bf16 [M, F] | None,
    h quantized | None, g and u quantized ([2, M, F]) | None) as asked for by ``bf16``, ``quantized``, ``checkpoint``."""
    if w.parts != 2:
        raise ValueError("the gated layer takes the stacked (gate, up) weights: parts = 2")
    codes, scale, x, ldx, M = _activations(x, q, w.K, 1, w.codes, w.scale)
    F, dev, fb = w.N, w.codes.device, _blocks(w.N)
    h = torch.empty((M, F), dtype=torch.bfloat16, device=dev) if bf16 else None
    hq = gu = None
    if quantized:
        hq = Fp8Block(torch.empty((M, F), dtype=torch.uint8, device=dev),
                      torch.empty((fb, M), dtype=torch.float32, device=dev), _mode(mode) == SCALE_M1)
    if checkpoint:
        gu = Fp8Block(torch.empty((2, M, F), dtype=torch.uint8, device=dev),
                      torch.empty((2, fb, M), dtype=torch.float32, device=dev), _mode(mode) == SCALE_M1)
    workspace = _fp8_workspace(workspace, M, w.K, dev)
    _check(lib().zq_fp8_gated_linear(_ptr(codes), _ptr(scale), _ptr(x), ldx, _scales(mode, w, q), M, F, w.K, _ptr(w.codes),
                                     _ptr(w.scale), _act(act), _ptr(h), F, _ptr(hq and hq.codes), _ptr(hq and hq.scale),
                                     _ptr(gu and gu.codes), _ptr(gu and gu.scale), _ptr(workspace), workspace.numel(),
                                     _stream()), "zq_fp8_gated_linear")
    return h, hq, gu


def fp8_gated_linear_backward(wt: Fp8Weight, gu: Fp8Block, *, dy=None, q: Optional[Fp8Block] = None, act="silu",
                              mode="none", workspace: Optional[torch.Tensor] = None):
    """Gradients of g and u from the gradient of the block's output (bf16 ``dy`` or quantized ``q``), the transposed down
    projection ``wt`` and the checkpoint ``gu``.  Returns (bf16 [2, M, F], the same quantized)."""
    if wt.parts != 1:
        raise ValueError("the backward pass takes one transposed down projection: parts = 1")
    codes, scale, dy, lddy, M = _activations(dy, q, wt.K, 1, wt.codes, wt.scale, gu.codes, gu.scale)
    F, dev, fb = wt.N, wt.codes.device, _blocks(wt.N)
    if tuple(gu.codes.shape) != (2, M, F) or tuple(gu.scale.shape) != (2, fb, M):
        raise ValueError(f"the checkpoint {tuple(gu.codes.shape)} does not fit [2, {M}, {F}]")
    _expect(gu.codes, torch.uint8, "gu.codes")
    _expect(gu.scale, torch.float32, "gu.scale")
    d = torch.empty((2, M, F), dtype=torch.bfloat16, device=dev)
    dq = Fp8Block(torch.empty((2, M, F), dtype=torch.uint8, device=dev),
                  torch.empty((2, fb, M), dtype=torch.float32, device=dev), _mode(mode) == SCALE_M1)
    workspace = _fp8_workspace(workspace, M, wt.K, dev)
    _check(lib().zq_fp8_gated_linear_backward(_ptr(codes), _ptr(scale), _ptr(dy), lddy, _scales(mode, wt, q), M, F, wt.K,
                                              _ptr(wt.codes), _ptr(wt.scale), _act(act), _ptr(gu.codes),
                                              _ptr(gu.scale), _ptr(d), _ptr(dq.codes), _ptr(dq.scale),
                                              _ptr(workspace), workspace.numel(), _stream()),
           "zq_fp8_gated_linear_backward")
    return d, dq


def fp8_weight_grad(g: torch.Tensor, q: Fp8Block, *, out_dtype=torch.float32,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW = g^T x^ with the checkpoint ``q`` of x.  g: bf16 [M, N] (row stride allowed) -> [N, K]; or contiguous
    [parts, M, N] -> [parts, N, K]."""
    dwdt = _out_type(out_dtype)
    parts = g.shape[0] if g.dim() == 3 else 1
    g0 = g[0] if g.dim() == 3 else g
    ldg, M, N = _rows(g0, "g")
    K = q.codes.shape[-1]
    codes, scale, _, _, Mq = _activations(None, q, K, 1, g)
    if Mq != M:
        raise ValueError(f"g has {M} rows, the checkpoint {Mq}")
    dw = g.new_empty((parts, N, K) if g.dim() == 3 else (N, K), dtype=out_dtype)
    workspace = _fp8_workspace(workspace, 0, 16, g.device)
    _check(lib().zq_fp8_weight_grad(_ptr(g), ldg, g.stride(0) if g.dim() == 3 else 0, parts, _ptr(codes), _ptr(scale),
                                    M, N, K, _ptr(dw), dwdt, _ptr(workspace), workspace.numel(), _stream()), "zq_fp8_weight_grad")
    return dw


def fp8_gated_ffn_saved_bytes(M: int, K: int, F: int) -> int:
    return int(lib().zq_fp8_gated_ffn_saved_bytes(M, K, F))


def fp8_gated_ffn_workspace_bytes(M: int, K: int, F: int, N: int, training: bool = False) -> int:
    return int(lib().zq_fp8_gated_ffn_workspace_bytes(M, K, F, N, 1 if training else 0))


def fp8_gated_ffn(gate_up: Fp8Weight, down: Fp8Weight, x: torch.Tensor, *, act="silu", mode="none",
                  out_dtype=torch.bfloat16, save=False, workspace: torch.Tensor):
    """The gated feed-forward block in one call: y = (act(x Wg^T) * (x Wu^T)) Wd^T.  With ``save`` returns (y, the uint8
    buffer that :func:`fp8_gated_ffn_backward` reads), else y."""
    ydt = _out_type(out_dtype)
    ldx, M, K = _rows(x, "x")
    F, N = gate_up.N, down.N
    if gate_up.parts != 2 or down.parts != 1 or gate_up.K != K or down.K != F:
        raise ValueError(f"x [{M}, {K}], gate_up {gate_up.parts} x [{F}, {gate_up.K}] and down [{N}, {down.K}] do not belong "
                         "together")
    _expect(workspace, torch.uint8, "workspace")
    _on_gpu(x, gate_up.codes, gate_up.scale, down.codes, down.scale, workspace)
    y = torch.empty((M, N), dtype=out_dtype, device=x.device)
    saved = torch.empty((fp8_gated_ffn_saved_bytes(M, K, F),), dtype=torch.uint8, device=x.device) if save else None
    _check(lib().zq_fp8_gated_ffn(x.data_ptr(), ldx, _ffn_scales(mode, gate_up, down), M, K, F, N, gate_up.codes.data_ptr(),
                                  gate_up.scale.data_ptr(), down.codes.data_ptr(), down.scale.data_ptr(), _act(act),
                                  y.data_ptr(), ydt, N, _ptr(saved),
                                  workspace.data_ptr(), workspace.numel(), _stream()), "zq_fp8_gated_ffn")
    return (y, saved) if save else y


def fp8_gated_ffn_backward(gate_up_t: Fp8Weight, down_t: Fp8Weight, dy: torch.Tensor, saved: torch.Tensor, *, act="silu",
                           mode="none", out_dtype=torch.bfloat16, workspace: torch.Tensor):
    """(dx [M, K], dW of (gate, up) [2, F, K], dW of down [N, F]) from dy bf16 [M, N], the transposed weights and what
    :func:`fp8_gated_ffn` saved."""
    dt = _out_type(out_dtype)
    lddy, M, N = _rows(dy, "dy")
    F, K = down_t.N, gate_up_t.N
    if gate_up_t.parts != 2 or down_t.parts != 1 or gate_up_t.K != F or down_t.K != N:
        raise ValueError(f"dy [{M}, {N}], gate_up_t {gate_up_t.parts} x [{K}, {gate_up_t.K}] and down_t [{F}, {down_t.K}] do "
                         "not belong together")
    _expect(saved, torch.uint8, "saved")
    if saved.numel() != fp8_gated_ffn_saved_bytes(M, K, F):
        raise ValueError(f"what was saved ({saved.numel()} bytes) is not of {M} tokens")
    _expect(workspace, torch.uint8, "workspace")
    _on_gpu(dy, saved, gate_up_t.codes, gate_up_t.scale, down_t.codes, down_t.scale, workspace)
    dev = dy.device
    dx = torch.empty((M, K), dtype=out_dtype, device=dev)
    dwgu = torch.empty((2, F, K), dtype=out_dtype, device=dev)
    dwd = torch.empty((N, F), dtype=out_dtype, device=dev)
    _check(lib().zq_fp8_gated_ffn_backward(dy.data_ptr(), lddy,
                                           _ffn_scales(mode, gate_up_t, down_t), M, K, F, N, saved.data_ptr(),
                                           gate_up_t.codes.data_ptr(), gate_up_t.scale.data_ptr(),
                                           down_t.codes.data_ptr(), down_t.scale.data_ptr(), _act(act), dx.data_ptr(),
                                           dwgu.data_ptr(), dwd.data_ptr(),
                                           dt, workspace.data_ptr(),
                                           workspace.numel(), _stream()), "zq_fp8_gated_ffn_backward")
    return dx, dwgu, dwd
