"""Python binding of the dense feed-forward block's C ABI (include/weave_ffn.h).

Argument marshalling only, as for the MoE layer: every product and rounding runs inside the CUDA library; PyTorch is
used for device memory and streams.  There is no CPU or eager fallback.

`stream`: the number (cuda_stream) of the stream that a call runs on; by default the device's current one.  Inputs have to be
ready there, and results that the call allocates belong to that stream, as if it had been made the current one.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import WeaveError, WEAVE_OK, _check, _empty, load as _load_library

BF16, F32, INT8 = 0, 1, 2

EXPORTS = [
    "weave_ffn_workspace_bytes", "weave_ffn_create", "weave_ffn_forward", "weave_ffn_backward", "weave_ffn_status",
    "weave_ffn_set_timeout_ms", "weave_ffn_debug_plan", "weave_ffn_debug_withhold_arrival", "weave_ffn_last_cuda_error", "weave_ffn_destroy",
    "weave_int8_quantize", "weave_int8_linear_workspace_bytes", "weave_int8_linear_create",
    "weave_int8_linear_forward", "weave_int8_linear_status", "weave_int8_linear_set_timeout_ms",
    "weave_int8_linear_debug_plan", "weave_int8_linear_last_cuda_error", "weave_int8_linear_destroy",
]


class _FfnConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int), ("ffn", ctypes.c_int), ("max_tokens", ctypes.c_int),
                ("weight_type", ctypes.c_int), ("backward", ctypes.c_int),
                ("gate_up", ctypes.c_void_p), ("down", ctypes.c_void_p),
                ("gate_up_scale", ctypes.c_void_p), ("down_scale", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class _Int8LinearConfig(ctypes.Structure):
    _fields_ = [("in_features", ctypes.c_int), ("out_features", ctypes.c_int), ("max_tokens", ctypes.c_int),
                ("weight", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class _Product(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("kernel", "mma_n", "tail_n", "width", "parts", "blocks", "tiles", "mn_run", "mn_atom")]


_lib = None


def load():
    """The package's library with these prototypes declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _load_library()
    vp, ci, vpp = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_void_p)
    lib.weave_ffn_workspace_bytes.restype = ctypes.c_size_t
    lib.weave_ffn_workspace_bytes.argtypes = [ctypes.POINTER(_FfnConfig)]
    lib.weave_int8_linear_workspace_bytes.restype = ctypes.c_size_t
    lib.weave_int8_linear_workspace_bytes.argtypes = [ctypes.POINTER(_Int8LinearConfig)]
    for name, args in (("weave_ffn_create", [ctypes.POINTER(_FfnConfig), vpp]),
                       ("weave_ffn_forward", [vp, vp, vp, ci, vp]),
                       ("weave_ffn_backward", [vp, vp, vp, vp, vp, vp, ci, vp]),
                       ("weave_ffn_status", [vp]), ("weave_ffn_set_timeout_ms", [vp, ci]),
                       ("weave_ffn_debug_plan", [ctypes.POINTER(_FfnConfig), ci, ci, ci, ctypes.POINTER(_Product), ci]),
                       ("weave_ffn_debug_withhold_arrival", [vp, ci]),
                       ("weave_ffn_last_cuda_error", [vp]), ("weave_ffn_destroy", [vp]),
                       ("weave_int8_quantize", [vp, ci, ci, ci, vp, vp, vp]),
                       ("weave_int8_linear_create", [ctypes.POINTER(_Int8LinearConfig), vpp]),
                       ("weave_int8_linear_forward", [vp, vp, ci, vp, vp, ci, ci, vp]),
                       ("weave_int8_linear_status", [vp]), ("weave_int8_linear_set_timeout_ms", [vp, ci]),
                       ("weave_int8_linear_debug_plan",
                        [ctypes.POINTER(_Int8LinearConfig), ci, ci, ci, ctypes.POINTER(_Product), ci]),
                       ("weave_int8_linear_last_cuda_error", [vp]), ("weave_int8_linear_destroy", [vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = ci, args
    _lib = lib
    return lib


def ffn_workspace_bytes(hidden: int, ffn: int, max_tokens: int, int8: bool = False, backward: bool = False) -> int:
    """Device scratch of a block's handle; 0 for a shape that it does not take."""
    cfg = _FfnConfig(hidden, ffn, max_tokens, INT8 if int8 else BF16, int(backward))
    return int(load().weave_ffn_workspace_bytes(ctypes.byref(cfg)))


def int8_linear_workspace_bytes(in_features: int, out_features: int, max_tokens: int) -> int:
    cfg = _Int8LinearConfig(in_features, out_features, max_tokens)
    return int(load().weave_int8_linear_workspace_bytes(ctypes.byref(cfg)))


def _products(fn, *args):
    out = (_Product * 5)()
    n = fn(*args, out, 5)
    if n < 0:
        raise WeaveError(n, fn.__name__)
    return [{name: getattr(p, name) for name, _ in _Product._fields_} for p in out[:n]]


def ffn_plan(hidden: int, ffn: int, T: int, max_tokens: Optional[int] = None, int8: bool = False, backward: bool = False,
             n_sm: int = 148):
    """How a call is carried out, one dict per product (see weave_ffn_debug_plan); needs no GPU."""
    cfg = _FfnConfig(hidden, ffn, max_tokens or T, INT8 if int8 else BF16, int(backward))
    return _products(load().weave_ffn_debug_plan, ctypes.byref(cfg), int(backward), T, n_sm)


def int8_linear_plan(in_features: int, out_features: int, T: int, max_tokens: Optional[int] = None, x_type: int = BF16,
                     n_sm: int = 148):
    cfg = _Int8LinearConfig(in_features, out_features, max_tokens or T)
    return _products(load().weave_int8_linear_debug_plan, ctypes.byref(cfg), x_type, T, n_sm)


_types = {}


def _type_of(dtype):
    if not _types:
        import torch
        _types.update({torch.bfloat16: BF16, torch.float32: F32, torch.int8: INT8})
    return _types[dtype]


def quantize_rows(x, q=None, scale=None, stream: Optional[int] = None):
    """x [rows, cols] in bf16 or fp32 -> (int8 [rows, cols], fp32 scale [rows]): scale = max|row| / 127, the nearest
    integer to x / scale.  Tokens' activations and weights' output channels alike (see weave_int8_quantize)."""
    import torch
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous() and x.dtype in (torch.bfloat16, torch.float32)
    rows, cols = x.shape
    if q is None:
        q = _empty((rows, cols), torch.int8, x.device, stream)
    if scale is None:
        scale = _empty((rows,), torch.float32, x.device, stream)
    assert q.device == x.device and q.dtype == torch.int8 and q.is_contiguous() and tuple(q.shape) == (rows, cols)
    assert scale.device == x.device and scale.dtype == torch.float32 and scale.is_contiguous() and tuple(scale.shape) == (rows,)
    if stream is None:
        stream = torch.cuda.current_stream(x.device).cuda_stream
    with torch.cuda.device(x.device):
        _check(load().weave_int8_quantize(x.data_ptr(), _type_of(x.dtype), rows, cols, q.data_ptr(), scale.data_ptr(), stream),
               "weave_int8_quantize")
    return q, scale


class _Handle:
    """What the classes below share: the workspace, the handle, its status and its end."""

    _name = ""       # prefix of the C calls

    def _open(self, cfg, nbytes: int, device):
        import torch
        if nbytes == 0:
            raise WeaveError(-1, f"{self._name}_workspace_bytes")
        self._torch, self._lib, self.device = torch, load(), device
        self.workspace = torch.empty(nbytes + 1024, dtype=torch.uint8, device=device)
        cfg.workspace = self.workspace.data_ptr() + (-self.workspace.data_ptr()) % 1024
        cfg.workspace_bytes = nbytes
        self._h = ctypes.c_void_p()
        self._index = device.index
        self._raw_stream = torch._C._cuda_getCurrentRawStream      # current_stream() without the object around it: 4 us less
        with torch.cuda.device(device):
            _check(getattr(self._lib, f"{self._name}_create")(ctypes.byref(cfg), ctypes.byref(self._h)), f"{self._name}_create")

    def _call(self, fn, *args, stream: Optional[int]):
        if stream is None:
            stream = self._raw_stream(self._index)
        if self._torch.cuda.current_device() == self._index:
            rc = fn(self._h, *args, stream)
        else:
            with self._torch.cuda.device(self.device):
                rc = fn(self._h, *args, stream)
        if rc != WEAVE_OK:
            raise WeaveError(rc, fn.__name__)

    def status(self) -> int:
        """Waits for all work on the device; 0, or ERR_TIMEOUT after a wait that gave up, and clears it."""
        with self._torch.cuda.device(self.device):
            return int(getattr(self._lib, f"{self._name}_status")(self._h))

    def check(self):
        st = self.status()
        if st != WEAVE_OK:
            raise WeaveError(st, "device status")

    def set_timeout_ms(self, ms: int):
        _check(getattr(self._lib, f"{self._name}_set_timeout_ms")(self._h, ms), f"{self._name}_set_timeout_ms")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._torch.cuda.synchronize(self.device)
            getattr(self._lib, f"{self._name}_destroy")(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _need_cuda(what: str):
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError(f"{what} needs a CUDA device (sm_100); there is no CPU path")
    return torch


class GatedFFN(_Handle):
    """The dense block down(silu(gate x) * (up x)) in bf16: gate_up [2I, H] (gate rows, then up rows), down [H, I], on
    the GPU.  backward=True reserves what backward() needs (6 T I bytes instead of 2 T I).

    No operator of autograd: forward()'s result carries no graph, whatever x or the weights require, and backward() is called
    by the training step itself; it overwrites its results, so that gradients of several micro-batches are added up outside."""

    _name = "weave_ffn"

    def __init__(self, gate_up, down, max_tokens: int = 4096, backward: bool = False):
        torch = _need_cuda("GatedFFN")
        assert gate_up.is_cuda and gate_up.dtype == torch.bfloat16 and gate_up.is_contiguous() and gate_up.dim() == 2
        assert down.device == gate_up.device and down.dtype == torch.bfloat16 and down.is_contiguous()
        twoI, H = gate_up.shape
        assert twoI % 2 == 0 and tuple(down.shape) == (H, twoI // 2)
        self.H, self.I, self.max_tokens = H, twoI // 2, max_tokens
        self.gate_up, self.down = gate_up, down
        cfg = _FfnConfig(H, self.I, max_tokens, BF16, int(backward), gate_up.data_ptr(), down.data_ptr(), None, None)
        self._open(cfg, ffn_workspace_bytes(H, self.I, max_tokens, backward=backward), gate_up.device)

    def _rows(self, *tensors):
        T = tensors[0].shape[0]
        for t in tensors:
            assert t.device == self.device and t.dtype == self._torch.bfloat16 and t.is_contiguous()
            assert tuple(t.shape) == (T, self.H)
        return T

    def forward(self, x, out=None, stream: Optional[int] = None):
        """x bf16 [T, H] -> bf16 [T, H]."""
        if out is None:
            out = self._torch.empty_like(x) if stream is None else _empty(x.shape, x.dtype, self.device, stream)
        T = self._rows(x, out)
        self._call(self._lib.weave_ffn_forward, x.data_ptr(), out.data_ptr(), T, stream=stream)
        return out

    def debug_withhold_arrival(self, cta: int):
        _check(self._lib.weave_ffn_debug_withhold_arrival(self._h, cta), "weave_ffn_debug_withhold_arrival")

    def backward(self, x, dy, dx=None, dgate_up=None, ddown=None, stream: Optional[int] = None):
        """(dx [T, H], dgate_up [2I, H], ddown [H, I]) in bf16 for the gradient dy of forward(x); all overwritten."""
        torch = self._torch
        if stream is None:       # (3 us less in a call than by _empty())
            dx = torch.empty_like(x) if dx is None else dx
            dgate_up = torch.empty_like(self.gate_up) if dgate_up is None else dgate_up
            ddown = torch.empty_like(self.down) if ddown is None else ddown
        else:
            dx, dgate_up, ddown = (_empty(like.shape, like.dtype, self.device, stream) if g is None else g
                                   for g, like in ((dx, x), (dgate_up, self.gate_up), (ddown, self.down)))
        T = self._rows(x, dy, dx)
        for g, w in ((dgate_up, self.gate_up), (ddown, self.down)):
            assert g.device == self.device and g.dtype == torch.bfloat16 and g.is_contiguous() and g.shape == w.shape
        self._call(self._lib.weave_ffn_backward, x.data_ptr(), dy.data_ptr(), dx.data_ptr(), dgate_up.data_ptr(), ddown.data_ptr(),
                   T, stream=stream)
        return dx, dgate_up, ddown


class Int8FFN(_Handle):
    """The block with weights in 8-bit integers: gate_up int8 [2I, H] with fp32 scales [2I], down int8 [H, I] with fp32
    scales [H] (quantize_rows() of the bf16 weights); x and the result are bf16."""

    _name = "weave_ffn"

    def __init__(self, gate_up, gate_up_scale, down, down_scale, max_tokens: int = 4096):
        torch = _need_cuda("Int8FFN")
        assert gate_up.is_cuda and gate_up.dtype == torch.int8 and gate_up.is_contiguous() and gate_up.dim() == 2
        assert down.device == gate_up.device and down.dtype == torch.int8 and down.is_contiguous()
        twoI, H = gate_up.shape
        assert twoI % 2 == 0 and tuple(down.shape) == (H, twoI // 2)
        for s, n in ((gate_up_scale, twoI), (down_scale, H)):
            assert s.device == gate_up.device and s.dtype == torch.float32 and s.is_contiguous() and tuple(s.shape) == (n,)
        self.H, self.I, self.max_tokens = H, twoI // 2, max_tokens
        self.gate_up, self.gate_up_scale, self.down, self.down_scale = gate_up, gate_up_scale, down, down_scale
        cfg = _FfnConfig(H, self.I, max_tokens, INT8, 0, gate_up.data_ptr(), down.data_ptr(), gate_up_scale.data_ptr(),
                         down_scale.data_ptr())
        self._open(cfg, ffn_workspace_bytes(H, self.I, max_tokens, int8=True), gate_up.device)

    _rows = GatedFFN._rows
    forward = GatedFFN.forward
    debug_withhold_arrival = GatedFFN.debug_withhold_arrival


class Int8Linear(_Handle):
    """y = x W^T with W in 8-bit integers [N, K] and one fp32 scale per output channel [N]; x either bf16 or fp32
    (rounded to 8 bits with one scale per token) or already int8 with its scales."""

    _name = "weave_int8_linear"

    def __init__(self, weight, scale, max_tokens: int = 4096):
        torch = _need_cuda("Int8Linear")
        assert weight.is_cuda and weight.dtype == torch.int8 and weight.is_contiguous() and weight.dim() == 2
        self.N, self.K = weight.shape
        assert scale.device == weight.device and scale.dtype == torch.float32 and scale.is_contiguous()
        assert tuple(scale.shape) == (self.N,)
        self.max_tokens, self.weight, self.scale = max_tokens, weight, scale
        cfg = _Int8LinearConfig(self.K, self.N, max_tokens, weight.data_ptr(), scale.data_ptr())
        self._open(cfg, int8_linear_workspace_bytes(self.K, self.N, max_tokens), weight.device)

    def forward(self, x, x_scale=None, out=None, out_dtype=None, stream: Optional[int] = None):
        """x [T, K] in bf16, fp32 or (with x_scale fp32 [T]) int8 -> [T, N] in out_dtype (bf16 by default, or fp32)."""
        torch = self._torch
        T = x.shape[0]
        if out is None:
            dtype = out_dtype or torch.bfloat16
            out = torch.empty(T, self.N, dtype=dtype, device=self.device) if stream is None else _empty((T, self.N), dtype, self.device, stream)
        assert x.device == self.device and x.is_contiguous() and tuple(x.shape) == (T, self.K)
        assert x.dtype in (torch.bfloat16, torch.float32, torch.int8) and (x.dtype == torch.int8) == (x_scale is not None)
        if x_scale is not None:
            assert x_scale.device == self.device and x_scale.dtype == torch.float32 and x_scale.is_contiguous()
            assert tuple(x_scale.shape) == (T,)
        assert out.device == self.device and out.is_contiguous() and tuple(out.shape) == (T, self.N)
        assert out.dtype in (torch.bfloat16, torch.float32) and out_dtype in (None, out.dtype)
        self._call(self._lib.weave_int8_linear_forward, x.data_ptr(), _type_of(x.dtype),
                   None if x_scale is None else x_scale.data_ptr(), out.data_ptr(), _type_of(out.dtype), T, stream=stream)
        return out
