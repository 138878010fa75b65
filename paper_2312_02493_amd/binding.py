"""ctypes binding of libartopk.so.  Same names as the C ABI; marshalling only.

PyTorch is used for device memory (tensor.data_ptr()) and for the stream handle;
no step of the compressor runs in PyTorch.
"""

from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))

ARTOPK_STAR, ARTOPK_VAR, ARTOPK_FIXED, ARTOPK_VAR_TOPK, ARTOPK_VAR_G = 0, 1, 2, 3, 4
ARTOPK_STAR_COUNTER = 5
ARTOPK_G_F32, ARTOPK_G_BF16, ARTOPK_G_F16 = 0, 1, 2
ARTOPK_OPT_GUESS_MIN_N, ARTOPK_OPT_UPDATE_TILES_MIN_N, ARTOPK_OPT_LEADER_FIRST, ARTOPK_OPT_NONTEMPORAL = 0, 1, 2, 3
ARTOPK_OPT_STAGE_TILES, ARTOPK_OPT_SHORT_MAX_N = 4, 5
ARTOPK_PRODUCTS_HALF, ARTOPK_PRODUCTS_SPLIT, ARTOPK_PRODUCTS_DEFAULT = 0, 1, -1
ARTOPK_MAX_TOP = 64
PROF_NAMES = ("pass_a", "select", "gather", "update", "total")

_SYMBOLS = (
    "artopk_create", "artopk_destroy", "artopk_last_error", "artopk_status", "artopk_variance",
    "artopk_select_topk", "artopk_gather_sum", "artopk_scatter_residual", "artopk_step",
    "artopk_set_profile", "artopk_get_profile", "artopk_version", "artopk_compression_gain",
    "artopk_apply_update", "artopk_topk_workers", "artopk_select_info", "artopk_step_g16",
    "artopk_set_option", "artopk_get_option", "artopk_variance_static", "artopk_set_step_counter",
    "artopk_scratch_bytes",
    "artopk_norm_create", "artopk_norm_scratch_bytes", "artopk_norm_destroy", "artopk_norm_last_error",
    "artopk_layernorm_forward", "artopk_layernorm_backward",
    "artopk_matrices_create", "artopk_matrices_scratch_bytes", "artopk_matrices_info", "artopk_matrices_destroy",
    "artopk_matrices_last_error", "artopk_orthogonalize", "artopk_muon_step",
    "artopk_tokens_create", "artopk_tokens_scratch_bytes", "artopk_tokens_destroy", "artopk_tokens_last_error",
    "artopk_tokens_status", "artopk_embedding_forward", "artopk_embedding_backward", "artopk_token_logprobs",
    "artopk_token_logprobs_backward",
    "artopk_adamw_create", "artopk_adamw_scratch_bytes", "artopk_adamw_state_elems", "artopk_adamw_destroy",
    "artopk_adamw_last_error", "artopk_adamw_step", "artopk_adamw_set_step", "artopk_adamw_values",
)


class ArTopkError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"artopk error {code}: {text}")
        self.code = code


def lib_path() -> str:
    return os.path.join(HERE, "libartopk.so")


def exported_symbols():
    return _SYMBOLS


_lib = None


def load_library():
    """Load libartopk.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2312_02493_amd.build`")
    lib = C.CDLL(path)
    vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    lib.artopk_create.argtypes = [C.POINTER(vp), i32, i64, i64, i32, vp]
    lib.artopk_destroy.argtypes = [vp]
    lib.artopk_last_error.argtypes = [vp]
    lib.artopk_status.argtypes = [vp]
    lib.artopk_variance.argtypes = [vp, vp, i32, i64, vp, vp]
    lib.artopk_select_topk.argtypes = [vp, vp, i64, i32, vp, vp, i64, vp]
    lib.artopk_gather_sum.argtypes = [vp, vp, i32, i64, vp, i64, vp, vp]
    lib.artopk_scatter_residual.argtypes = [vp, vp, i32, i64, vp, i64, vp, vp]
    lib.artopk_step.argtypes = [vp, vp, vp, i32, i64, i32, vp, vp, i64, i32, u64, i32, vp, vp, vp, vp, vp, vp]
    lib.artopk_step_g16.argtypes = [vp, vp, i32, vp, i32, i64, i32, vp, vp, i64, i32, u64, i32, vp, vp, vp, vp, vp,
                                    vp]
    lib.artopk_topk_workers.argtypes = [vp, vp, i32, i64, i64, vp, vp, vp, vp]
    lib.artopk_compression_gain.argtypes = [vp, vp, i32, i64, vp, i64, vp]
    lib.artopk_apply_update.argtypes = [vp, vp, i64, vp, vp, i64, C.c_float]
    lib.artopk_set_profile.argtypes = [vp, i32]
    lib.artopk_get_profile.argtypes = [vp, C.POINTER(C.c_float), i32]
    lib.artopk_select_info.argtypes = [vp, C.POINTER(i32), i32]
    lib.artopk_set_option.argtypes = [vp, i32, i64]
    lib.artopk_get_option.argtypes = [vp, i32, C.POINTER(i64)]
    lib.artopk_variance_static.argtypes = [vp, i32, i64, vp, vp, vp]
    lib.artopk_set_step_counter.argtypes = [vp, C.c_uint64]
    lib.artopk_scratch_bytes.argtypes = [i32, i64, i64, i32]
    f32 = C.c_float
    lib.artopk_norm_create.argtypes = [C.POINTER(vp), i64, i64, vp]
    lib.artopk_norm_scratch_bytes.argtypes = [i64, i64]
    lib.artopk_norm_destroy.argtypes = [vp]
    lib.artopk_norm_last_error.argtypes = [vp]
    lib.artopk_layernorm_forward.argtypes = [vp, vp, i64, i32, i64, i64, vp, vp, f32, vp, i64, vp, vp]
    lib.artopk_layernorm_backward.argtypes = [vp, vp, i64, vp, i64, i32, i64, i64, vp, vp, vp, vp, i64, vp, vp, i32, i32]
    lib.artopk_matrices_create.argtypes = [C.POINTER(vp), vp, i32, i64, i32, i32, vp]
    lib.artopk_matrices_scratch_bytes.argtypes = [vp, i32, i64, i32, i32]
    lib.artopk_matrices_info.argtypes = [vp, i32, i64, i32, i32, i32, vp, i32]
    lib.artopk_matrices_destroy.argtypes = [vp]
    lib.artopk_matrices_last_error.argtypes = [vp]
    lib.artopk_orthogonalize.argtypes = [vp, vp, vp, i32, vp, f32]
    lib.artopk_muon_step.argtypes = [vp, vp, vp, vp, f32, f32, i32, f32, f32, f32, i32, vp, f32]
    f64 = C.c_double
    lib.artopk_tokens_create.argtypes = [C.POINTER(vp), i64, i64, i64, vp]
    lib.artopk_tokens_scratch_bytes.argtypes = [i64, i64, i64]
    for name in ("artopk_tokens_destroy", "artopk_tokens_last_error", "artopk_tokens_status", "artopk_adamw_destroy",
                 "artopk_adamw_last_error"):
        getattr(lib, name).argtypes = [vp]
    lib.artopk_embedding_forward.argtypes = [vp, vp, i64, i32, i64, i64, vp, i32, i64, f32, vp, i64, i32]
    lib.artopk_embedding_backward.argtypes = [vp, vp, i64, i32, vp, i32, i64, i64, f32, vp, i64, i32, i64, i32]
    lib.artopk_token_logprobs.argtypes = [vp, vp, i64, i32, i64, i64, vp, i32, f32, vp, vp, vp, vp, i32, vp, vp]
    lib.artopk_token_logprobs_backward.argtypes = [vp, vp, i64, i32, i64, i64, vp, i32, f32, vp, vp, vp, vp, vp, vp, vp, i64]
    lib.artopk_adamw_create.argtypes = [C.POINTER(vp), vp, i32, i64, i32, i32, vp]
    lib.artopk_adamw_scratch_bytes.argtypes = [vp, i32, i64]
    lib.artopk_adamw_state_elems.argtypes = [vp, i32, i64]
    lib.artopk_adamw_step.argtypes = [vp, vp, vp, vp, vp, vp, i64, f32, f32, f64, f64, f32, u64]
    lib.artopk_adamw_set_step.argtypes = [vp, i64]
    lib.artopk_adamw_values.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.artopk_version.restype = i32
    for name in _SYMBOLS:
        if name.endswith(("_scratch_bytes", "_state_elems")):
            getattr(lib, name).restype = i64
        elif name.endswith("_last_error"):
            getattr(lib, name).restype = C.c_char_p
        elif name != "artopk_version":
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _ptr_table(tensors: Sequence):
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = int(t.data_ptr())
    return arr


def _i64_array(values):
    if values is None:
        return None
    arr = (C.c_int64 * len(values))()
    for i, v in enumerate(values):
        arr[i] = int(v)
    return arr


def artopk_scratch_bytes(max_w: int, max_n: int, max_k: int, max_segments: int = 1) -> int:
    """Device bytes a Context of these limits allocates (-1: limits refused); needs no GPU."""
    return int(load_library().artopk_scratch_bytes(int(max_w), int(max_n), int(max_k), int(max_segments)))


def artopk_variance_static(x: Sequence, var_out, argmax_out=None, stream: Optional[int] = None):
    """The context-free variance call that allocates nothing (enqueued on `stream`, default: torch's current)."""
    import torch

    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = lib.artopk_variance_static(_ptr_table(x), len(x), x[0].numel(), _ptr(var_out), _ptr(argmax_out),
                                    C.c_void_p(stream))
    if rc != 0:
        raise ArTopkError(rc, lib.artopk_last_error(None).decode())


class Context:
    """Owns one artopk_ctx bound to the current torch stream of the current device."""

    def __init__(self, max_w: int, max_n: int, max_k: int, max_segments: int = 1, stream: Optional[int] = None):
        import torch

        if not torch.cuda.is_available():
            raise RuntimeError("the AR-Topk library needs a GPU; there is no CPU path")
        self._lib = load_library()
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self._h = C.c_void_p()
        rc = self._lib.artopk_create(C.byref(self._h), max_w, max_n, max_k, max_segments, C.c_void_p(stream))
        if rc != 0:
            raise ArTopkError(rc, "artopk_create failed")

    # -- plumbing ------------------------------------------------------------
    def _check(self, rc: int):
        if rc != 0:
            raise ArTopkError(rc, self._lib.artopk_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.artopk_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def status(self):
        self._check(self._lib.artopk_status(self._h))

    def set_profile(self, level: int):
        """0 off, 1 events around pass A only, 2 events at every stage boundary."""
        self._check(self._lib.artopk_set_profile(self._h, int(level)))

    def set_option(self, key: int, value: int):
        self._check(self._lib.artopk_set_option(self._h, int(key), int(value)))

    def set_step_counter(self, value: int):
        self._check(self._lib.artopk_set_step_counter(self._h, int(value)))

    def get_option(self, key: int) -> int:
        out = C.c_int64()
        self._check(self._lib.artopk_get_option(self._h, int(key), C.byref(out)))
        return int(out.value)

    def select_info(self) -> dict:
        buf = (C.c_int32 * 10)()
        self._check(self._lib.artopk_select_info(self._h, buf, 10))
        return {"guessed": int(buf[0]), "from_mask": int(buf[1]), "list_count": int(buf[2]),
                "list_level": int(buf[3]), "dominant_workers": int(buf[4]), "short": int(buf[5]), "many": int(buf[6]),
                "one_launch": int(buf[7]), "tiles": int(buf[8]), "tile_bounds": int(buf[9])}

    def get_profile(self) -> dict:
        buf = (C.c_float * len(PROF_NAMES))()
        self._check(self._lib.artopk_get_profile(self._h, buf, len(PROF_NAMES)))
        return {name: float(buf[i]) for i, name in enumerate(PROF_NAMES)}

    # -- the five entry points ---------------------------------------------
    def artopk_variance(self, x: Sequence, var_out, argmax_out=None):
        n = x[0].numel()
        self._check(self._lib.artopk_variance(self._h, _ptr_table(x), len(x), n, _ptr(var_out), _ptr(argmax_out)))

    def artopk_select_topk(self, acc, k: int, idx_out, seg_off=None, seg_k=None):
        nseg = 1 if seg_off is None else len(seg_k)
        self._check(self._lib.artopk_select_topk(self._h, _ptr(acc), acc.numel(), nseg, _i64_array(seg_off),
                                                 _i64_array(seg_k), k, _ptr(idx_out)))

    def artopk_gather_sum(self, acc: Sequence, idx, k: int, vals_out, sum_out):
        n = acc[0].numel()
        self._check(self._lib.artopk_gather_sum(self._h, _ptr_table(acc), len(acc), n, _ptr(idx), k,
                                                _ptr(vals_out), _ptr(sum_out)))

    def artopk_scatter_residual(self, residual: Sequence, idx, k: int, summed, update):
        n = residual[0].numel()
        self._check(self._lib.artopk_scatter_residual(self._h, _ptr_table(residual), len(residual), n, _ptr(idx), k,
                                                      _ptr(summed), _ptr(update)))

    def artopk_topk_workers(self, acc: Sequence, k: int, idx_out, vals_out=None, sqnorm_out=None, argmax_out=None):
        n = acc[0].numel()
        self._check(self._lib.artopk_topk_workers(self._h, _ptr_table(acc), len(acc), n, k, _ptr(idx_out),
                                                  _ptr(vals_out), _ptr(sqnorm_out), _ptr(argmax_out)))

    def artopk_compression_gain(self, residual: Sequence, vals, k: int, gain_out):
        n = residual[0].numel()
        self._check(self._lib.artopk_compression_gain(self._h, _ptr_table(residual), len(residual), n, _ptr(vals),
                                                      k, _ptr(gain_out)))

    def artopk_apply_update(self, weights, idx, summed, k: int, eta: float):
        self._check(self._lib.artopk_apply_update(self._h, _ptr(weights), weights.numel(), _ptr(idx), _ptr(summed),
                                                  k, C.c_float(eta)))

    def artopk_step(self, g: Sequence, residual: Sequence, k: int, mode: int, step: int, idx_out, sum_out,
                    update_out, vals_out=None, leader_out=None, var_out=None, fixed_leader: int = 0,
                    seg_off=None, seg_k=None):
        n = g[0].numel()
        nseg = 1 if seg_off is None else len(seg_k)
        self._check(self._lib.artopk_step(self._h, _ptr_table(g), _ptr_table(residual), len(g), n, nseg,
                                          _i64_array(seg_off), _i64_array(seg_k), k, mode, step, fixed_leader,
                                          _ptr(leader_out), _ptr(var_out), _ptr(idx_out), _ptr(vals_out),
                                          _ptr(sum_out), _ptr(update_out)))

    def artopk_step_g16(self, g: Sequence, g_type: int, residual: Sequence, k: int, mode: int, step: int, idx_out,
                        sum_out, update_out, vals_out=None, leader_out=None, var_out=None, fixed_leader: int = 0,
                        seg_off=None, seg_k=None):
        n = g[0].numel()
        nseg = 1 if seg_off is None else len(seg_k)
        self._check(self._lib.artopk_step_g16(self._h, _ptr_table(g), g_type, _ptr_table(residual), len(g), n, nseg,
                                              _i64_array(seg_off), _i64_array(seg_k), k, mode, step, fixed_leader,
                                              _ptr(leader_out), _ptr(var_out), _ptr(idx_out), _ptr(vals_out),
                                              _ptr(sum_out), _ptr(update_out)))


_types = {}  # torch's element types -> ARTOPK_G_*, filled when torch is there
_whole = {}  # torch's types of whole numbers -> bits, the same


def _elem_types():
    if not _types:
        import torch

        _types.update({torch.float32: ARTOPK_G_F32, torch.bfloat16: ARTOPK_G_BF16, torch.float16: ARTOPK_G_F16})
        _whole.update({torch.uint8: 8, torch.int32: 32, torch.int64: 64})
    return _types


def _elem_type(t) -> int:
    """ARTOPK_G_* of a tensor's elements."""
    kind = _elem_types().get(t.dtype)
    if kind is None:
        raise ArTopkError(-1, f"elements of type {t.dtype} are not taken")
    return kind


def _rows(t, name: str, device: int):
    """(address, distance of rows, rows, cols) of a matrix on the device whose columns lie side by side."""
    if t.get_device() != device:
        raise ArTopkError(-1, f"{name} is on {t.device}, not on the handle's device {device}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2:
        raise ArTopkError(-1, f"{name} has {len(shape)} dimensions, not 2")
    rows, cols = shape
    if stride[1] != 1 and cols > 1:
        raise ArTopkError(-1, f"{name}'s columns do not lie side by side")
    return t.data_ptr(), (stride[0] if rows > 1 else cols), rows, cols


def _vector(t, name: str, length: int, device: int, kind: Optional[int] = None) -> Optional[int]:
    """Address of a contiguous vector of `length` elements (of type `kind`) on the device, or None for None."""
    if t is None:
        return None
    if t.get_device() != device:
        raise ArTopkError(-1, f"{name} is on {t.device}, not on the handle's device {device}")
    if t.numel() != length or not t.is_contiguous():
        raise ArTopkError(-1, f"{name} is not a contiguous vector of {length} elements")
    if kind is not None and _types.get(t.dtype) != kind:
        raise ArTopkError(-1, f"{name} is {t.dtype}, which is not what is taken")
    return t.data_ptr()


def _coefficients(steps: int, coefficients):
    """steps x 3 floats from None, one (a, b, c) for all steps, or one for each."""
    if coefficients is None:
        return None
    rows = [coefficients] * steps if len(coefficients) == 3 and not hasattr(coefficients[0], "__len__") else coefficients
    if len(rows) != steps or any(len(r) != 3 for r in rows):
        raise ArTopkError(-1, f"coefficients are not (a, b, c) or {steps} of these")
    return (C.c_float * (3 * max(steps, 1)))(*[float(v) for r in rows for v in r])


class _Handle:
    """A library handle bound to the current torch stream of the current device."""

    _name = ""

    def _open(self, stream: Optional[int], *args):
        import torch

        if not torch.cuda.is_available():
            raise RuntimeError("the AR-Topk library needs a GPU; there is no CPU path")
        self._lib = load_library()
        _elem_types()
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self._device = torch.cuda.current_device()
        h = C.c_void_p()
        rc = getattr(self._lib, f"artopk_{self._name}_create")(C.byref(h), *args, C.c_void_p(stream))
        if rc != 0:
            raise ArTopkError(rc, self._lib.artopk_last_error(None).decode())
        self._h = h

    def _check(self, rc: int):
        if rc != 0:
            raise ArTopkError(rc, getattr(self._lib, f"artopk_{self._name}_last_error")(self._h).decode())

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            getattr(self._lib, f"artopk_{self._name}_destroy")(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def artopk_norm_scratch_bytes(max_rows: int, max_cols: int) -> int:
    """Device bytes a NormContext of these limits allocates (-1: limits refused); needs no GPU."""
    return int(load_library().artopk_norm_scratch_bytes(int(max_rows), int(max_cols)))


class NormContext(_Handle):
    """Owns one artopk_norm: layer norms of up to max_rows rows of up to max_cols elements."""

    _name = "norm"

    def __init__(self, max_rows: int, max_cols: int, stream: Optional[int] = None):
        self._open(stream, int(max_rows), int(max_cols))

    def artopk_layernorm_forward(self, x, gamma, beta, y, mean_out=None, rstd_out=None, eps: float = 1e-5):
        dev = self._device
        px, sx, rows, cols = _rows(x, "x", dev)
        py, sy, rows_y, cols_y = _rows(y, "y", dev)
        if rows_y != rows or cols_y != cols or y.dtype != x.dtype:
            raise ArTopkError(-1, "y's shape or type is not x's")
        self._check(self._lib.artopk_layernorm_forward(
            self._h, px, sx, _elem_type(x), rows, cols, _vector(gamma, "gamma", cols, dev, ARTOPK_G_F32),
            _vector(beta, "beta", cols, dev, ARTOPK_G_F32), eps, py, sy,
            _vector(mean_out, "mean_out", rows, dev, ARTOPK_G_F32), _vector(rstd_out, "rstd_out", rows, dev, ARTOPK_G_F32)))

    def artopk_layernorm_backward(self, dy, x, gamma, mean, rstd, dx, dgamma=None, dbeta=None, accumulate: bool = False):
        dev = self._device
        px, sx, rows, cols = _rows(x, "x", dev)
        pd, sd, rows_d, cols_d = _rows(dy, "dy", dev)
        if rows_d != rows or cols_d != cols or dy.dtype != x.dtype:
            raise ArTopkError(-1, "dy's shape or type is not x's")
        po, so = None, cols
        if dx is not None:
            po, so, rows_d, cols_d = _rows(dx, "dx", dev)
            if rows_d != rows or cols_d != cols or dx.dtype != x.dtype:
                raise ArTopkError(-1, "dx's shape or type is not x's")
        grad = dbeta if dgamma is None else dgamma
        if dgamma is not None and dbeta is not None and dgamma.dtype != dbeta.dtype:
            raise ArTopkError(-1, "dgamma and dbeta are of different types")
        self._check(self._lib.artopk_layernorm_backward(
            self._h, pd, sd, px, sx, _elem_type(x), rows, cols, _vector(gamma, "gamma", cols, dev, ARTOPK_G_F32),
            _vector(mean, "mean", rows, dev, ARTOPK_G_F32), _vector(rstd, "rstd", rows, dev, ARTOPK_G_F32), po, so,
            _vector(dgamma, "dgamma", cols, dev), _vector(dbeta, "dbeta", cols, dev),
            ARTOPK_G_F32 if grad is None else _elem_type(grad), int(accumulate)))


class _Matrix(C.Structure):
    _fields_ = [("offset", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("scale", C.c_float)]


def _matrix_table(matrices: Sequence):
    table = (_Matrix * max(1, len(matrices)))()
    for i, m in enumerate(matrices):
        offset, rows, cols = (int(v) for v in m[:3])
        table[i] = _Matrix(offset, rows, cols, float(m[3]) if len(m) > 3 else 1.0)
    return table


def artopk_matrices_scratch_bytes(matrices: Sequence, n: int, elem_type: int = ARTOPK_G_F32,
                                  products: int = ARTOPK_PRODUCTS_DEFAULT) -> int:
    """Device bytes a MatrixContext of these arguments allocates (-1: refused); needs no GPU."""
    return int(load_library().artopk_matrices_scratch_bytes(_matrix_table(matrices), len(matrices), int(n),
                                                            int(elem_type), int(products)))


def artopk_matrices_info(matrices: Sequence, n: int, elem_type: int = ARTOPK_G_F32, products: int = ARTOPK_PRODUCTS_DEFAULT,
                         weights: bool = False) -> list:
    """The groups of launches of a MatrixContext of these arguments, as dicts; needs no GPU."""
    lib = load_library()
    out = (C.c_int32 * 17)()
    rc = lib.artopk_matrices_info(_matrix_table(matrices), len(matrices), int(n), int(elem_type), int(products), int(weights), out,
                                  len(out))
    if rc != 0:
        raise ArTopkError(rc, lib.artopk_last_error(None).decode())
    names = ("matrices", "parts", "one_launch", "pairs", "gram_tile", "square_tile", "apply_tile", "shared_tiles")
    return [dict(zip(names, out[1 + 8 * i:9 + 8 * i])) for i in range(out[0])]


class MatrixContext(_Handle):
    """Owns one artopk_matrices: matrices (offset, rows, cols[, scale]) of a flat vector of n elements."""

    _name = "matrices"

    def __init__(self, matrices: Sequence, n: int, elem_type: int = ARTOPK_G_F32, products: int = ARTOPK_PRODUCTS_DEFAULT,
                 stream: Optional[int] = None):
        self.n, self.elem_type = int(n), int(elem_type)
        self._open(stream, _matrix_table(matrices), len(matrices), self.n, self.elem_type, int(products))

    def _flat(self, t, name: str) -> Optional[int]:
        if t is not None and _elem_type(t) != self.elem_type:
            raise ArTopkError(-1, f"{name} is {t.dtype}, which is not the handle's type")
        return _vector(t, name, self.n, self._device)

    def artopk_orthogonalize(self, x, out, steps: int = 5, coefficients=None, eps: float = 1e-7):
        self._check(self._lib.artopk_orthogonalize(self._h, self._flat(x, "x"), self._flat(out, "out"), int(steps),
                                                   _coefficients(int(steps), coefficients), eps))

    def artopk_muon_step(self, weights, momentum, update, eta: float, mu: float = 0.95, nesterov: bool = True,
                         decay: float = 0.0, eta_rest: float = 0.0, update_scale: float = 1.0, steps: int = 5,
                         coefficients=None, eps: float = 1e-7):
        self._check(self._lib.artopk_muon_step(
            self._h, self._flat(weights, "weights"), _vector(momentum, "momentum", self.n, self._device, ARTOPK_G_F32),
            _vector(update, "update", self.n, self._device, ARTOPK_G_F32), update_scale, mu, int(nesterov),
            eta, decay, eta_rest, int(steps), _coefficients(int(steps), coefficients),
            eps))


def artopk_tokens_scratch_bytes(max_tokens: int, max_vocab: int, max_width: int = 1) -> int:
    """Device bytes a TokenContext of these limits allocates (-1: limits refused); needs no GPU."""
    return int(load_library().artopk_tokens_scratch_bytes(int(max_tokens), int(max_vocab), int(max_width)))


def _token_bits(t) -> int:
    bits = _whole.get(t.dtype, 0)
    if bits < 32:
        raise ArTopkError(-1, f"tokens are {t.dtype}: int32 or int64 are taken")
    return bits


def _top_rows(t, name: str, rows: int, top: int, device: int, right: bool) -> int:
    """Address of a contiguous rows x top matrix of the right type on the device."""
    if t.get_device() != device:
        raise ArTopkError(-1, f"{name} is on {t.device}, not on the handle's device {device}")
    if tuple(t.shape) != (rows, top) or not t.is_contiguous() or not right:
        raise ArTopkError(-1, f"{name}, {t.dtype} {tuple(t.shape)}, is not a contiguous {rows} x {top} matrix of what is taken")
    return t.data_ptr()


class TokenContext(_Handle):
    """Owns one artopk_tokens: embedding rows and log probabilities of up to max_tokens tokens of up to max_vocab."""

    _name = "tokens"

    def __init__(self, max_tokens: int, max_vocab: int, max_width: int = 1, stream: Optional[int] = None):
        self._open(stream, int(max_tokens), int(max_vocab), int(max_width))

    def status(self):
        self._check(self._lib.artopk_tokens_status(self._h))

    def artopk_embedding_forward(self, table, tokens, y, scale: float = 1.0):
        dev = self._device
        pt, st, vocab, width = _rows(table, "table", dev)
        py, sy, count, width_y = _rows(y, "y", dev)
        if width_y != width:
            raise ArTopkError(-1, "y's rows are not as long as table's")
        self._check(self._lib.artopk_embedding_forward(
            self._h, pt, st, _elem_type(table), vocab, width, _vector(tokens, "tokens", count, dev), _token_bits(tokens), count,
            scale, py, sy, _elem_type(y)))

    def artopk_embedding_backward(self, dy, tokens, dtable, scale: float = 1.0, accumulate: bool = False):
        dev = self._device
        pd, sd, count, width = _rows(dy, "dy", dev)
        pt, st, vocab, width_t = _rows(dtable, "dtable", dev)
        if width_t != width:
            raise ArTopkError(-1, "dtable's rows are not as long as dy's")
        self._check(self._lib.artopk_embedding_backward(
            self._h, pd, sd, _elem_type(dy), _vector(tokens, "tokens", count, dev), _token_bits(tokens), count, width, scale, pt,
            st, _elem_type(dtable), vocab, int(accumulate)))

    def artopk_token_logprobs(self, logits, tokens=None, logp_out=None, peak_out=None, logsum_out=None, entropy_out=None,
                              top_ids_out=None, top_logp_out=None, scale: float = 1.0):
        dev = self._device
        p, s, rows, vocab = _rows(logits, "logits", dev)
        top, ids, lps = 0, None, None
        if top_ids_out is not None or top_logp_out is not None:
            if top_ids_out is None or top_logp_out is None or len(top_ids_out.shape) != 2:
                raise ArTopkError(-1, "top_ids_out and top_logp_out are not two matrices")
            top = top_ids_out.shape[1]
            ids = _top_rows(top_ids_out, "top_ids_out", rows, top, dev, _whole.get(top_ids_out.dtype) == 32)
            lps = _top_rows(top_logp_out, "top_logp_out", rows, top, dev, _types.get(top_logp_out.dtype) == ARTOPK_G_F32)
        self._check(self._lib.artopk_token_logprobs(
            self._h, p, s, _elem_type(logits), rows, vocab, _vector(tokens, "tokens", rows, dev),
            32 if tokens is None else _token_bits(tokens), scale, _vector(logp_out, "logp_out", rows, dev, ARTOPK_G_F32),
            _vector(peak_out, "peak_out", rows, dev, ARTOPK_G_F32), _vector(logsum_out, "logsum_out", rows, dev, ARTOPK_G_F32),
            _vector(entropy_out, "entropy_out", rows, dev, ARTOPK_G_F32), top, ids, lps))

    def artopk_token_logprobs_backward(self, logits, tokens, peak, logsum, dlogits, dlogp=None, dlse=None, entropy=None,
                                       dentropy=None, scale: float = 1.0):
        dev = self._device
        p, s, rows, vocab = _rows(logits, "logits", dev)
        pd, sd, rows_d, vocab_d = _rows(dlogits, "dlogits", dev)
        if rows_d != rows or vocab_d != vocab or dlogits.dtype != logits.dtype:
            raise ArTopkError(-1, "dlogits' shape or type is not logits'")
        kind = _elem_type(logits)
        f = [_vector(t, name, rows, dev, ARTOPK_G_F32) for t, name in (
            (peak, "peak"), (logsum, "logsum"), (entropy, "entropy"), (dlogp, "dlogp"), (dlse, "dlse"), (dentropy, "dentropy"))]
        self._check(self._lib.artopk_token_logprobs_backward(
            self._h, p, s, kind, rows, vocab, _vector(tokens, "tokens", rows, dev), 32 if tokens is None else _token_bits(tokens),
            scale, *f, pd, sd))


class _Tensor(C.Structure):
    _fields_ = [("offset", C.c_int64), ("count", C.c_int64), ("eta_scale", C.c_float), ("decay", C.c_float)]


def _tensor_table(tensors: Sequence):
    table = (_Tensor * max(1, len(tensors)))()
    for i, t in enumerate(tensors):
        table[i] = _Tensor(int(t[0]), int(t[1]), float(t[2]) if len(t) > 2 else 1.0, float(t[3]) if len(t) > 3 else 0.0)
    return table


def artopk_adamw_scratch_bytes(tensors: Sequence, n: int) -> int:
    """Device bytes an AdamWContext of these arguments allocates (-1: refused); needs no GPU."""
    return int(load_library().artopk_adamw_scratch_bytes(_tensor_table(tensors), len(tensors), int(n)))


def artopk_adamw_state_elems(tensors: Sequence, n: int) -> int:
    """Elements of each moment (-1: refused); with 8 bits a byte each, and two bytes of scales for every 256; needs no GPU."""
    return int(load_library().artopk_adamw_state_elems(_tensor_table(tensors), len(tensors), int(n)))


class AdamWContext(_Handle):
    """Owns one artopk_adamw: tensors (offset, count[, eta_scale[, decay]]) of a flat vector of n elements."""

    _name = "adamw"

    def __init__(self, tensors: Sequence, n: int, elem_type: int = ARTOPK_G_F32, state_bits: int = 32,
                 stream: Optional[int] = None):
        self.n, self.elem_type, self.state_bits = int(n), int(elem_type), int(state_bits)
        table = _tensor_table(tensors)
        self._open(stream, table, len(tensors), self.n, self.elem_type, self.state_bits)
        self.state_elems = int(self._lib.artopk_adamw_state_elems(table, len(tensors), self.n))

    def new_state(self):
        """(first, second, scales) before the first step, on the handle's device; scales is None with 32 bits."""
        import torch

        dev = torch.device("cuda", self._device)
        kind = torch.uint8 if self.state_bits == 8 else torch.float32
        first, second = (torch.zeros(self.state_elems, dtype=kind, device=dev) for _ in range(2))
        return first, second, torch.zeros(self.state_elems // 256, 2, dtype=kind, device=dev) if self.state_bits == 8 else None

    def _moments(self, first, second, scales):
        eight = self.state_bits == 8
        out = []
        for t, name, length, codes in ((first, "first", self.state_elems, eight), (second, "second", self.state_elems, eight),
                                       (scales, "scales", self.state_elems // 128, True)):
            if t is not None and (_whole.get(t.dtype) != 8 if codes else _types.get(t.dtype) != ARTOPK_G_F32):
                raise ArTopkError(-1, f"{name} is {t.dtype}, which is not what is taken")
            out.append(_vector(t, name, length, self._device))
        return out

    def set_step(self, step: int):
        self._check(self._lib.artopk_adamw_set_step(self._h, int(step)))

    def artopk_adamw_step(self, weights, update, first, second, scales=None, step: int = 0, eta: float = 1e-3,
                          beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, update_scale: float = 1.0, seed: int = 0):
        if _elem_type(weights) != self.elem_type:
            raise ArTopkError(-1, f"weights is {weights.dtype}, which is not the handle's type")
        self._check(self._lib.artopk_adamw_step(
            self._h, _vector(weights, "weights", self.n, self._device), _vector(update, "update", self.n, self._device, ARTOPK_G_F32),
            *self._moments(first, second, scales), int(step), update_scale, eta, beta1, beta2, eps, int(seed) & (1 << 64) - 1))

    def artopk_adamw_values(self, first, second, scales, first_out=None, second_out=None):
        outs = [t for t in (first_out, second_out) if t is not None]
        kinds = {_elem_type(t) for t in outs}
        if len(kinds) > 1:
            raise ArTopkError(-1, "first_out and second_out are of different types")
        self._check(self._lib.artopk_adamw_values(
            self._h, *self._moments(first, second, scales), kinds.pop() if kinds else ARTOPK_G_F32,
            *[_vector(t, name, self.state_elems, self._device) for t, name in ((first_out, "first_out"), (second_out, "second_out"))]))
