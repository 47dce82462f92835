"""ctypes binding of libmodse.so: the same calls as include/modse.h.

Argument marshalling only - every step of the layer runs in the library's CUDA
kernels.  PyTorch tensors are used as device buffers; their ``data_ptr()`` and
the current CUDA stream are handed to the C ABI.  There is no CPU fallback:
loading fails with an error if the shared library has not been built.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libmodse.so")

MODSE_OK = 0
MODSE_ERR_INVALID_ARG = 1
MODSE_ERR_UNSUPPORTED = 2
MODSE_ERR_WORKSPACE_TOO_SMALL = 3
MODSE_ERR_STATE = 4
MODSE_ERR_CUDA = 5
MODSE_ERR_DEVICE_TIMEOUT = 6
MODSE_ERR_DEVICE_BOUNDS = 7
MODSE_F32 = 0
MODSE_BF16 = 1
MODSE_E4M3 = 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
N_STAGES = 12
MODSE_FUSE_GATHER = 1
MODSE_FUSE_DG_ROWDOT = 2
MODSE_FUSE_SCATTER = 4
DEFAULT_TILE_PLAN = 0x3F3A         # every product on CTA pairs; fallback: products 1, 3, 4, 5 on one-CTA 256-row tiles
PAIR_SHIFT = 8                     # bit 8 + k of a plan: product k on 256-row tiles computed by a pair of CTAs


class ModseError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


class _Weights(ctypes.Structure):
    _fields_ = [("w_router", ctypes.c_void_p), ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p),
                ("w_down", ctypes.c_void_p)]


class _WGrads(ctypes.Structure):
    _fields_ = [("dw_router", ctypes.c_void_p), ("dw_gate", ctypes.c_void_p), ("dw_up", ctypes.c_void_p),
                ("dw_down", ctypes.c_void_p)]


class _Linear(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "w", "x_scale", "w_scale", "bias", "residual", "z", "y")]


class _LinearGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "w", "dy", "z", "dx", "dw", "dbias")]


class _Matrix(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("update", ctypes.c_void_p), ("ld_grad", ctypes.c_longlong),
                ("ld_update", ctypes.c_longlong), ("rows", ctypes.c_int), ("cols", ctypes.c_int), ("scale", ctypes.c_float)]


_lib = None
torch = None      # bound by the first call that is handed tensors: loading and the host-side calls do without it


def _bind_torch():
    global torch
    import torch as module
    torch = module


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load libmodse.so (raises if it is missing: there is no other path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} not found: build it with `python -m paper_2409_12210_b200.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    ip = ctypes.POINTER(ctypes.c_int)
    lib.modse_create.restype = vp
    lib.modse_create.argtypes = [ci, ci, ip, ci]
    lib.modse_last_create_error.restype = ci
    lib.modse_destroy.restype = ci
    lib.modse_destroy.argtypes = [vp]
    lib.modse_check_pairs.restype = ci
    lib.modse_check_pairs.argtypes = [ip, ci, ip]
    lib.modse_status_string.restype = ctypes.c_char_p
    lib.modse_status_string.argtypes = [ci]
    lib.modse_workspace_bytes.restype = sz
    lib.modse_workspace_bytes.argtypes = [vp, ci, ci, ci]
    lib.modse_forward.restype = ci
    lib.modse_forward.argtypes = [vp, ci, ctypes.POINTER(_Weights), vp, ci, vp, vp, sz, ci, vp]
    lib.modse_backward.restype = ci
    lib.modse_backward.argtypes = [vp, ci, ctypes.POINTER(_Weights), vp, vp, ci, vp, ctypes.POINTER(_WGrads), vp, sz,
                                   vp]
    pp = ctypes.POINTER(ctypes.c_void_p)
    lib.modse_get_routing.restype = ci
    lib.modse_get_routing.argtypes = [vp, vp, ci, pp, pp, pp, pp, pp, pp, pp]
    lib.modse_get_gate_grads.restype = ci
    lib.modse_get_gate_grads.argtypes = [vp, vp, ci, pp, pp]
    lib.modse_check_device_status.restype = ci
    lib.modse_check_device_status.argtypes = [vp, vp, vp]
    lib.modse_last_launch_count.restype = ci
    lib.modse_last_launch_count.argtypes = [vp]
    lib.modse_route_static_scratch.restype = ci
    lib.modse_route_static_scratch.argtypes = [ci, ci, ci, ci, vp, vp, ci, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.modse_route_static_scratch_capacity.restype = sz
    lib.modse_route_static_scratch_status.restype = ci
    lib.modse_route_static_scratch_status.argtypes = [vp]
    lib.modse_aux_loss.restype = ci
    lib.modse_aux_loss.argtypes = [vp, vp, ci, ctypes.c_float, vp, vp, vp, vp]
    lib.modse_set_aux_loss.restype = ci
    lib.modse_set_aux_loss.argtypes = [vp, ctypes.c_float]
    lib.modse_set_noise_gate.restype = ci
    lib.modse_set_noise_gate.argtypes = [vp, vp, ctypes.c_float, ctypes.c_float]
    lib.modse_set_noise_grads.restype = ci
    lib.modse_set_noise_grads.argtypes = [vp, vp, vp]
    lib.modse_tune_forward.restype = ci
    lib.modse_tune_forward.argtypes = [vp, ci, ctypes.POINTER(_Weights), vp, ci, vp, vp, sz, ci, vp]
    lib.modse_get_tile_plan.restype = ci
    lib.modse_get_tile_plan.argtypes = [vp]
    lib.modse_set_tile_plan.restype = ci
    lib.modse_set_tile_plan.argtypes = [vp, ci]
    lib.modse_set_output_f32.restype = ci
    lib.modse_set_output_f32.argtypes = [vp, ci]
    lib.modse_stage_timing_begin.restype = ci
    lib.modse_stage_timing_begin.argtypes = [vp, ci]
    lib.modse_stage_timing_end.restype = ci
    lib.modse_stage_timing_end.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ip]
    lib.modse_stage_name.restype = ctypes.c_char_p
    lib.modse_stage_name.argtypes = [ci]
    lib.modse_debug_set_default_tile_plan.restype = None
    lib.modse_debug_set_default_tile_plan.argtypes = [ci]
    lib.modse_debug_set_dynamic_tiles.restype = None
    lib.modse_debug_set_dynamic_tiles.argtypes = [ci]
    lib.modse_debug_set_epilogue_warps.restype = None
    lib.modse_debug_set_epilogue_warps.argtypes = [ci, ci, ci]
    lib.modse_debug_set_wait_limit_ms.restype = None
    lib.modse_debug_set_wait_limit_ms.argtypes = [ci]
    lib.modse_debug_skip_tile_loads.restype = None
    lib.modse_debug_skip_tile_loads.argtypes = [ci, ci]
    lib.modse_debug_workspace_offsets.restype = ci
    lib.modse_debug_workspace_offsets.argtypes = [vp, ci, ci, ci, ctypes.POINTER(sz), ctypes.POINTER(sz), ip]
    lib.modse_set_debug_checks.restype = ci
    lib.modse_set_debug_checks.argtypes = [vp, ci]
    lib.modse_set_fusion.restype = ci
    lib.modse_set_fusion.argtypes = [vp, ci]
    lib.modse_get_fusion.restype = ci
    lib.modse_get_fusion.argtypes = [vp]
    cf = ctypes.c_float
    lib.modse_add_rms_norm.restype = ci
    lib.modse_add_rms_norm.argtypes = [ci, ci, ci, vp, vp, vp, cf, vp, vp, vp, vp, vp]
    lib.modse_add_rms_norm_backward_workspace_bytes.restype = sz
    lib.modse_add_rms_norm_backward_workspace_bytes.argtypes = [ci, ci]
    lib.modse_add_rms_norm_backward.restype = ci
    lib.modse_add_rms_norm_backward.argtypes = [ci, ci, ci, vp, vp, cf, vp, vp, vp, vp, vp, sz, vp]
    lib.modse_linear_workspace_bytes.restype = sz
    lib.modse_linear_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.modse_linear.restype = ci
    lib.modse_linear.argtypes = [ci, ci, ci, ci, ci, ctypes.POINTER(_Linear), vp, sz, vp]
    lib.modse_linear_backward_workspace_bytes.restype = sz
    lib.modse_linear_backward_workspace_bytes.argtypes = [ci, ci, ci]
    lib.modse_linear_backward.restype = ci
    lib.modse_linear_backward.argtypes = [ci, ci, ci, ci, ctypes.POINTER(_LinearGrads), vp, sz, vp]
    fp = ctypes.POINTER(ctypes.c_float)
    lib.modse_orthogonalize_workspace_bytes.restype = sz
    lib.modse_orthogonalize_workspace_bytes.argtypes = [ci, ctypes.POINTER(_Matrix)]
    lib.modse_orthogonalize.restype = ci
    lib.modse_orthogonalize.argtypes = [ci, ci, ctypes.POINTER(_Matrix), ci, fp, cf, vp, sz, vp]
    lib.modse_orthogonalize_wgrads_workspace_bytes.restype = sz
    lib.modse_orthogonalize_wgrads_workspace_bytes.argtypes = [vp]
    lib.modse_orthogonalize_wgrads.restype = ci
    lib.modse_orthogonalize_wgrads.argtypes = [vp, ci, ctypes.POINTER(_WGrads), ctypes.POINTER(_WGrads), fp, ci, fp, cf, vp,
                                               sz, vp]
    lib.modse_check_workspace_status.restype = ci
    lib.modse_check_workspace_status.argtypes = [vp, vp]
    lib.modse_debug_use_fma_path.restype = None
    lib.modse_debug_use_fma_path.argtypes = [ci]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().modse_status_string(int(status)).decode()


def route_static_scratch(x, w_router, top_k: int):
    """Routing tables of a batch through modse_route_static_scratch: no workspace, the
    library's built-in scratch array is used.  Returns a dict of freshly created output
    tensors (the outputs are the caller's; only the scratch is the library's)."""
    import torch
    T, d = x.shape
    N = w_router.shape[0]
    dev = x.device
    out = {
        "topk_idx": torch.empty((T, top_k), dtype=torch.int32, device=dev),
        "topk_gate": torch.empty((T, top_k), dtype=torch.float32, device=dev),
        "counts": torch.empty(N, dtype=torch.int32, device=dev),
        "counts_slot": torch.empty((top_k, N), dtype=torch.int32, device=dev),
        "offsets": torch.empty(N + 1, dtype=torch.int32, device=dev),
        "row_of": torch.empty((T, top_k), dtype=torch.int32, device=dev),
        "token_of": torch.empty(T * top_k, dtype=torch.int32, device=dev),
    }
    st = load().modse_route_static_scratch(
        _dtype_code(x), d, N, top_k, x.data_ptr(), w_router.data_ptr(), T, out["topk_idx"].data_ptr(),
        out["topk_gate"].data_ptr(), out["counts"].data_ptr(), out["counts_slot"].data_ptr(),
        out["offsets"].data_ptr(), out["row_of"].data_ptr(), out["token_of"].data_ptr(),
        ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    if st != MODSE_OK:
        raise ModseError(st, "modse_route_static_scratch")
    return out


def route_static_scratch_status() -> int:
    """Status word the last modse_route_static_scratch call on this device left (synchronises the stream)."""
    import torch
    return int(load().modse_route_static_scratch_status(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))


def stage_name(i: int) -> str:
    return load().modse_stage_name(int(i)).decode()


def debug_set_default_tile_plan(plan: int) -> None:
    load().modse_debug_set_default_tile_plan(int(plan))


def debug_set_dynamic_tiles(on: bool) -> None:
    load().modse_debug_set_dynamic_tiles(int(bool(on)))


def debug_set_epilogue_warps(mask_128: int = 0, mask_256: int = 5, mask_pair: int = 0) -> None:
    load().modse_debug_set_epilogue_warps(int(mask_128), int(mask_256), int(mask_pair))


def debug_set_wait_limit_ms(ms: int) -> None:
    load().modse_debug_set_wait_limit_ms(int(ms))


def debug_skip_tile_loads(product: int, tile: int) -> None:
    load().modse_debug_skip_tile_loads(int(product), int(tile))


def debug_use_fma_path(on: bool) -> None:
    load().modse_debug_use_fma_path(int(bool(on)))


def check_pairs(ffn_sizes):
    """(ok, pair_sum) for the adjacent-pair rule of Sec. 3.1, Eq. 5-6."""
    arr = (ctypes.c_int * len(ffn_sizes))(*ffn_sizes)
    out = ctypes.c_int(0)
    ok = load().modse_check_pairs(arr, len(ffn_sizes), ctypes.byref(out))
    return bool(ok), (out.value if ok else None)


def _dtype_code(t):
    if torch is None:
        _bind_torch()
    if t.dtype == torch.float32:
        return MODSE_F32
    if t.dtype == torch.bfloat16:
        return MODSE_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


# ---- operators around the layer ---------------------------------------------
# A call on a token or two takes a few microseconds on the GPU, so what these wrappers cost on the host is what such a
# call costs: devices are compared by index and the stream is asked for by device, without the objects torch wraps them in.
def _buffer(name, t, shape, dtype, device):
    """Device address of a tensor that has to have this shape, type and device index (None: a null pointer)."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on CUDA device {device}, "
                         f"got {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}")
    return t.data_ptr()


def _current_stream(name, t):
    """(raw current stream, device index) of t's device, which has to be the current CUDA device."""
    if torch is None:
        _bind_torch()
    device = t.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: expected a tensor on the current CUDA device, got one on {t.device}")
    return torch._C._cuda_getCurrentRawStream(device), device


_INT_MAX = 2 ** 31 - 1


def _rows(name, t):
    shape = t.shape
    if len(shape) != 2 or shape[0] > _INT_MAX or shape[1] > _INT_MAX:      # ctypes would cut longer extents down silently
        raise ValueError(f"{name}: expected two dimensions of less than 2^31, got shape {tuple(shape)}")
    return shape


def add_rms_norm(x, residual, weight, eps: float, *, sum_out=None, y=None, y8=None, y_scale=None) -> None:
    """modse_add_rms_norm on the current stream: ``sum_out = x + residual`` and its root-mean-square norm times
    ``weight`` into ``y`` and, in 8 bits (torch.float8_e4m3fn) with one fp32 scale a row, into ``y8`` and ``y_scale``.
    ``residual`` and ``weight`` may be None, and so may any output the caller does not want."""
    T, d = shape = _rows("x", x)
    dt, code = x.dtype, _dtype_code(x)
    stream, dev = _current_stream("x", x)
    st = load().modse_add_rms_norm(
        code, T, d, _buffer("x", x, shape, dt, dev), _buffer("residual", residual, shape, dt, dev),
        _buffer("weight", weight, (d,), dt, dev), eps, _buffer("sum_out", sum_out, shape, dt, dev),
        _buffer("y", y, shape, dt, dev), _buffer("y8", y8, shape, torch.float8_e4m3fn, dev),
        _buffer("y_scale", y_scale, (T,), torch.float32, dev), stream)
    if st != MODSE_OK:
        raise ModseError(st, "modse_add_rms_norm")


def add_rms_norm_backward_workspace_bytes(n_tokens: int, d_model: int) -> int:
    return int(load().modse_add_rms_norm_backward_workspace_bytes(n_tokens, d_model))


def add_rms_norm_backward(s, weight, eps: float, dy, dsum, dx, dweight=None, workspace=None) -> None:
    """modse_add_rms_norm_backward: ``s`` is the sum forward wrote, ``dsum`` (or None) the gradient that reaches it past
    the norm; ``dx`` receives the gradient of x and of the residual alike, ``dweight`` (fp32, or None) the weight's."""
    T, d = shape = _rows("s", s)
    dt, code = s.dtype, _dtype_code(s)
    stream, dev = _current_stream("s", s)
    st = load().modse_add_rms_norm_backward(
        code, T, d, _buffer("s", s, shape, dt, dev), _buffer("weight", weight, (d,), dt, dev), eps,
        _buffer("dy", dy, shape, dt, dev), _buffer("dsum", dsum, shape, dt, dev), _buffer("dx", dx, shape, dt, dev),
        _buffer("dweight", dweight, (d,), torch.float32, dev), *_workspace(workspace, dev), stream)
    if st != MODSE_OK:
        raise ModseError(st, "modse_add_rms_norm_backward")


def _linear_code(dtype):
    if torch is None:
        _bind_torch()
    if dtype == torch.bfloat16:
        return MODSE_BF16
    if dtype == torch.float8_e4m3fn:
        return MODSE_E4M3
    raise TypeError(f"unsupported dtype {dtype}")


def linear_workspace_bytes(dtype, n_tokens: int, d_in: int, d_out: int) -> int:
    return int(load().modse_linear_workspace_bytes(_linear_code(dtype), n_tokens, d_in, d_out))


def linear(x, w, y, workspace, *, bias=None, residual=None, activation: str = "none", z=None, x_scale=None,
           w_scale=None) -> None:
    """modse_linear on the current stream: ``y = act(x w^T + bias) + residual``, the pre-activation into ``z`` if given.
    x [T, d_in] and w [d_out, d_in] are bf16, or torch.float8_e4m3fn with one fp32 scale a row (``x_scale``,
    ``w_scale``); everything else is bf16."""
    T, k = _rows("x", x)
    n = _rows("w", w)[0]
    code = _linear_code(x.dtype)
    stream, dev = _current_stream("x", x)
    bf, f32, out = torch.bfloat16, torch.float32, (T, n)
    args = _Linear(_buffer("x", x, (T, k), x.dtype, dev), _buffer("w", w, (n, k), x.dtype, dev),
                   _buffer("x_scale", x_scale, (T,), f32, dev), _buffer("w_scale", w_scale, (n,), f32, dev),
                   _buffer("bias", bias, (n,), bf, dev), _buffer("residual", residual, out, bf, dev),
                   _buffer("z", z, out, bf, dev), _buffer("y", y, out, bf, dev))
    st = load().modse_linear(code, T, k, n, ACTIVATIONS[activation], args, *_workspace(workspace, dev), stream)
    if st != MODSE_OK:
        raise ModseError(st, "modse_linear")


def linear_backward_workspace_bytes(n_tokens: int, d_in: int, d_out: int) -> int:
    return int(load().modse_linear_backward_workspace_bytes(n_tokens, d_in, d_out))


def linear_backward(x, w, dy, z, activation: str, dx, dw, dbias, workspace) -> None:
    """modse_linear_backward: the gradients of :func:`linear` on bf16 operands from ``dy`` and the saved ``z`` (None where
    there is no activation) into ``dx``, ``dw`` (bf16) and ``dbias`` (fp32); any of the three may be None."""
    T, k = _rows("x", x)
    n = _rows("w", w)[0]
    stream, dev = _current_stream("x", x)
    bf = torch.bfloat16
    args = _LinearGrads(_buffer("x", x, (T, k), bf, dev), _buffer("w", w, (n, k), bf, dev),
                        _buffer("dy", dy, (T, n), bf, dev), _buffer("z", z, (T, n), bf, dev),
                        _buffer("dx", dx, (T, k), bf, dev), _buffer("dw", dw, (n, k), bf, dev),
                        _buffer("dbias", dbias, (n,), torch.float32, dev))
    st = load().modse_linear_backward(T, k, n, ACTIVATIONS[activation], args, *_workspace(workspace, dev), stream)
    if st != MODSE_OK:
        raise ModseError(st, "modse_linear_backward")


MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalize_workspace_bytes(shapes) -> int:
    """Workspace bytes for matrices of these (rows, cols)."""
    arr = (_Matrix * len(shapes))(*[_Matrix(None, None, c, c, r, c, 1.0) for r, c in shapes])
    return int(load().modse_orthogonalize_workspace_bytes(len(shapes), arr))


def _ld(name, t):
    r, c = _rows(name, t)
    ld = t.stride(0) if r > 1 else max(c, 1)
    if (c > 1 and t.stride(1) != 1) or ld < c:
        raise ValueError(f"{name}: expected rows of contiguous elements that do not overlap, got strides {t.stride()}")
    return ld


def orthogonalize(grads, updates, workspace, *, scales=None, steps: int = 5, coefficients=MUON_COEFFICIENTS,
                  eps: float = 1e-7) -> None:
    """modse_orthogonalize on the current stream: the Newton-Schulz iterate of each matrix of ``grads`` (all bf16 or all
    fp32; rows may be strided, so column blocks of a wider matrix work) times its entry of ``scales`` into the bf16
    matrix of the same place in ``updates``."""
    n = len(grads)
    if len(updates) != n or (scales is not None and len(scales) != n):
        raise ValueError(f"{n} gradients, {len(updates)} updates, {n if scales is None else len(scales)} scales")
    if n == 0 and workspace is None:
        return
    dt, code = (grads[0].dtype, _dtype_code(grads[0])) if n else (None, MODSE_BF16)
    stream, dev = _current_stream("grads", grads[0]) if n else _current_stream("workspace", workspace)
    arr = (_Matrix * n)()
    for i, (g, u, m) in enumerate(zip(grads, updates, arr)):
        if (g.dtype != dt or g.get_device() != dev or u.dtype != torch.bfloat16 or u.get_device() != dev or
                u.shape != g.shape):
            raise ValueError(f"matrix {i}: expected a {dt} gradient and a bf16 update of one shape on CUDA device {dev}, got "
                             f"{g.dtype} {tuple(g.shape)} on {g.device} and {u.dtype} {tuple(u.shape)} on {u.device}")
        m.ld_grad, m.ld_update = _ld(f"gradient {i}", g), _ld(f"update {i}", u)
        m.grad, m.update = g.data_ptr(), u.data_ptr()
        m.rows, m.cols = g.shape
        m.scale = 1.0 if scales is None else scales[i]
    st = load().modse_orthogonalize(code, n, arr, steps, (ctypes.c_float * 3)(*coefficients), eps,
                                    *_workspace(workspace, dev), stream)
    if st != MODSE_OK:
        raise ModseError(st, "modse_orthogonalize")


def check_workspace_status(workspace) -> int:
    """Status the last operator call on this workspace left (synchronises the current stream, which has to be the call's).
    Like the calls it wants the workspace on the current device: another device's stream would not have been waited for."""
    stream, dev = _current_stream("workspace", workspace)
    return int(load().modse_check_workspace_status(_workspace(workspace, dev)[0], stream))


def _workspace(t, device):
    """(address, bytes) of a workspace tensor."""
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on CUDA device {device}, got one on {t.device}")
    return t.data_ptr(), t.numel() * t.element_size()


class ModseLayer:
    """Thin owner of a ``modse_layer_t``; methods mirror the C calls."""

    def __init__(self, d_model: int, ffn_sizes, top_k: int):
        lib = load()
        self.d_model, self.ffn_sizes, self.top_k = int(d_model), [int(h) for h in ffn_sizes], int(top_k)
        self.n_experts = len(self.ffn_sizes)
        arr = (ctypes.c_int * self.n_experts)(*self.ffn_sizes)
        self._h = lib.modse_create(self.d_model, self.n_experts, arr, self.top_k)
        if not self._h:
            raise ModseError(lib.modse_last_create_error(), "modse_create")

    def destroy(self):
        if getattr(self, "_h", None):
            load().modse_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def workspace_bytes(self, dtype_code: int, n_tokens: int, save_for_backward: bool) -> int:
        return int(load().modse_workspace_bytes(self._h, dtype_code, n_tokens, int(save_for_backward)))

    def alloc_workspace(self, dtype, n_tokens: int, save_for_backward: bool, device="cuda"):
        import torch
        code = MODSE_F32 if dtype == torch.float32 else MODSE_BF16
        nbytes = self.workspace_bytes(code, n_tokens, save_for_backward)
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    @staticmethod
    def _stream():
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def forward(self, w_router, w_gate, w_up, w_down, x, y, workspace, save_for_backward: bool):
        """Enqueue modse_forward on the current stream; tensors are device buffers
        laid out as include/modse.h states (w_down is [d, S])."""
        w = _Weights(w_router.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
        st = load().modse_forward(self._h, _dtype_code(x), ctypes.byref(w), x.data_ptr(), x.shape[0], y.data_ptr(),
                                  workspace.data_ptr(), workspace.numel(), int(save_for_backward), self._stream())
        if st != MODSE_OK:
            raise ModseError(st, "modse_forward")

    def tune_forward(self, w_router, w_gate, w_up, w_down, x, y, workspace, save_for_backward: bool) -> int:
        """Time the kernel shapes of the forward products on this device (synchronises) and keep the fastest;
        returns the plan (see modse_get_tile_plan)."""
        w = _Weights(w_router.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
        st = load().modse_tune_forward(self._h, _dtype_code(x), ctypes.byref(w), x.data_ptr(), x.shape[0],
                                       y.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                       int(save_for_backward), self._stream())
        if st != MODSE_OK:
            raise ModseError(st, "modse_tune_forward")
        return self.tile_plan()

    def tile_plan(self) -> int:
        return int(load().modse_get_tile_plan(self._h))

    def set_tile_plan(self, plan: int) -> None:
        st = load().modse_set_tile_plan(self._h, int(plan))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_tile_plan")

    def backward(self, w_router, w_gate, w_up, w_down, x, dy, dx, dw_router, dw_gate, dw_up, dw_down, workspace):
        w = _Weights(w_router.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
        g = _WGrads(dw_router.data_ptr(), dw_gate.data_ptr(), dw_up.data_ptr(), dw_down.data_ptr())
        st = load().modse_backward(self._h, _dtype_code(x), ctypes.byref(w), x.data_ptr(), dy.data_ptr(), x.shape[0],
                                   dx.data_ptr(), ctypes.byref(g), workspace.data_ptr(), workspace.numel(),
                                   self._stream())
        if st != MODSE_OK:
            raise ModseError(st, "modse_backward")

    @staticmethod
    def _view(ptr, workspace, count, dtype):
        off = ptr - workspace.data_ptr()
        return workspace[off:off + count * 4].view(dtype)

    def get_routing(self, workspace, n_tokens: int):
        """Views into the workspace: dict of topk_idx, topk_gate, counts, counts_slot,
        offsets, row_of, token_of (valid until the workspace is reused)."""
        import torch
        ptrs = [ctypes.c_void_p() for _ in range(7)]
        st = load().modse_get_routing(self._h, workspace.data_ptr(), n_tokens, *[ctypes.byref(p) for p in ptrs])
        if st != MODSE_OK:
            raise ModseError(st, "modse_get_routing")
        k, N, T = self.top_k, self.n_experts, n_tokens
        v = lambda i, n, dt: self._view(ptrs[i].value, workspace, n, dt)
        return {
            "topk_idx": v(0, T * k, torch.int32).view(T, k),
            "topk_gate": v(1, T * k, torch.float32).view(T, k),
            "counts": v(2, N, torch.int32),
            "counts_slot": v(3, k * N, torch.int32).view(k, N),
            "offsets": v(4, N + 1, torch.int32),
            "row_of": v(5, T * k, torch.int32).view(T, k),
            "token_of": v(6, T * k, torch.int32),
        }

    def get_gate_grads(self, workspace, n_tokens: int):
        import torch
        a, b = ctypes.c_void_p(), ctypes.c_void_p()
        st = load().modse_get_gate_grads(self._h, workspace.data_ptr(), n_tokens, ctypes.byref(a), ctypes.byref(b))
        if st != MODSE_OK:
            raise ModseError(st, "modse_get_gate_grads")
        T, k = n_tokens, self.top_k
        return (self._view(a.value, workspace, T * k, torch.float32).view(T, k),
                self._view(b.value, workspace, T * k, torch.float32).view(T, k))

    def check_device_status(self, workspace) -> int:
        return int(load().modse_check_device_status(self._h, workspace.data_ptr(), self._stream()))

    def set_debug_checks(self, on: bool) -> None:
        st = load().modse_set_debug_checks(self._h, int(bool(on)))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_debug_checks")

    def set_fusion(self, flags: int) -> None:
        st = load().modse_set_fusion(self._h, int(flags))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_fusion")

    def fusion(self) -> int:
        return int(load().modse_get_fusion(self._h))

    def debug_workspace_offsets(self, dtype_code: int, n_tokens: int, save_for_backward: bool):
        """(byte offset of prow_of, byte offset of the guard block behind topk_idx, padded rows)."""
        a, b, c = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_int(0)
        st = load().modse_debug_workspace_offsets(self._h, dtype_code, n_tokens, int(save_for_backward),
                                                  ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
        if st != MODSE_OK:
            raise ModseError(st, "modse_debug_workspace_offsets")
        return int(a.value), int(b.value), int(c.value)

    def set_aux_loss(self, alpha: float) -> None:
        st = load().modse_set_aux_loss(self._h, float(alpha))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_aux_loss")

    def aux_loss(self, workspace, n_tokens: int, alpha: float):
        """(loss [1], f [N], P [N]) device tensors of the auxiliary load-balance loss (Eq. 7-10)."""
        import torch
        dev = workspace.device
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        f = torch.empty(self.n_experts, dtype=torch.float32, device=dev)
        P = torch.empty(self.n_experts, dtype=torch.float32, device=dev)
        st = load().modse_aux_loss(self._h, workspace.data_ptr(), n_tokens, float(alpha), loss.data_ptr(),
                                   f.data_ptr(), P.data_ptr(), self._stream())
        if st != MODSE_OK:
            raise ModseError(st, "modse_aux_loss")
        return loss, f, P

    def set_noise_gate(self, w_noise, gamma: float = 0.0, eps: float = 0.0) -> None:
        """Second term of the router logits (Eq. 2): w_noise is a device tensor [N,d] in the layer's dtype
        that the caller keeps alive, or None to switch the term off."""
        self._w_noise = w_noise
        st = load().modse_set_noise_gate(self._h, w_noise.data_ptr() if w_noise is not None else None,
                                         float(gamma), float(eps))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_noise_gate")

    def set_noise_grads(self, dw_noise, dgamma) -> None:
        """Device tensors that backward fills: dw_noise [N,d] fp32, dgamma [1] fp32."""
        self._noise_grads = (dw_noise, dgamma)
        st = load().modse_set_noise_grads(self._h, dw_noise.data_ptr() if dw_noise is not None else None,
                                          dgamma.data_ptr() if dgamma is not None else None)
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_noise_grads")

    def orthogonalize_workspace_bytes(self) -> int:
        return int(load().modse_orthogonalize_wgrads_workspace_bytes(self._h))

    def orthogonalize_wgrads(self, dw_gate, dw_up, dw_down, up_gate, up_up, up_down, workspace, *, scales=None,
                             steps: int = 5, coefficients=MUON_COEFFICIENTS, eps: float = 1e-7) -> None:
        """Orthogonalised updates of every expert's three matrices from the gradients :meth:`backward` wrote (bf16, or
        fp32 with :meth:`set_output_f32`) into bf16 tensors of the same layouts.  ``scales``: None or N x 3 numbers
        (gate, up, down of each expert)."""
        import torch
        dt = dw_gate.dtype
        stream, dev = _current_stream("dw_gate", dw_gate)
        S, d = sum(self.ffn_sizes), self.d_model
        wide, tall, bf = (d, S), (S, d), torch.bfloat16
        g = _WGrads(None, _buffer("dw_gate", dw_gate, tall, dt, dev), _buffer("dw_up", dw_up, tall, dt, dev),
                    _buffer("dw_down", dw_down, wide, dt, dev))
        u = _WGrads(None, _buffer("up_gate", up_gate, tall, bf, dev), _buffer("up_up", up_up, tall, bf, dev),
                    _buffer("up_down", up_down, wide, bf, dev))
        flat = None
        if scales is not None:
            rows = [[float(v) for v in row] for row in scales]
            if len(rows) != self.n_experts or any(len(row) != 3 for row in rows):
                raise ValueError(f"scales: expected {self.n_experts} x 3 numbers")
            flat = (ctypes.c_float * (3 * self.n_experts))(*[v for row in rows for v in row])
        st = load().modse_orthogonalize_wgrads(self._h, _dtype_code(dw_gate), g, u, flat, steps,
                                               (ctypes.c_float * 3)(*coefficients), eps, *_workspace(workspace, dev), stream)
        if st != MODSE_OK:
            raise ModseError(st, "modse_orthogonalize_wgrads")

    def set_output_f32(self, on: bool) -> None:
        st = load().modse_set_output_f32(self._h, int(bool(on)))
        if st != MODSE_OK:
            raise ModseError(st, "modse_set_output_f32")

    def stage_timing_begin(self, max_calls: int) -> None:
        st = load().modse_stage_timing_begin(self._h, int(max_calls))
        if st != MODSE_OK:
            raise ModseError(st, "modse_stage_timing_begin")

    def stage_timing_end(self, max_calls: int):
        """[calls, N_STAGES] array of stage times in ms (-1: stage not run by that call)."""
        import numpy as np
        buf = (ctypes.c_float * (max_calls * N_STAGES))()
        n = ctypes.c_int(0)
        st = load().modse_stage_timing_end(self._h, buf, ctypes.byref(n))
        if st != MODSE_OK:
            raise ModseError(st, "modse_stage_timing_end")
        return np.ctypeslib.as_array(buf).reshape(max_calls, N_STAGES)[:n.value].copy()

    def last_launch_count(self) -> int:
        return int(load().modse_last_launch_count(self._h))


def pack_weights(inputs, device="cuda"):
    """Device tensors in the library's layouts from per-expert host arrays:
    w_router [N,d], w_gate/w_up [S,d], w_down [d,S] (experts side by side)."""
    import numpy as np
    import torch
    dt = torch.float32 if inputs.cfg.dtype == "f32" else torch.bfloat16
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dt)
    return (to(inputs.w_router), to(np.concatenate(inputs.w_gate, 0)), to(np.concatenate(inputs.w_up, 0)),
            to(np.concatenate(inputs.w_down, 1)))
