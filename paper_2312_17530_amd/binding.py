"""ctypes binding of librsdgc.so: argument marshalling only.

Function names mirror the C ABI declared in ``include/rsdgc.h``.  Device buffers are
torch tensors (torch is used for device memory and streams only); their addresses are
handed to the library unchanged.  There is no CPU fallback: if the library has not been
built, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librsdgc.so")

RSDGC_OK, RSDGC_EINVAL, RSDGC_ENOMEM, RSDGC_EHIP, RSDGC_ETOOBIG = 0, -1, -2, -3, -4
RSDGC_STATIC_WORKSPACE_BYTES = 64 << 20
RSDGC_MAX_P = 7

EXPORTS = [
    "rsdgc_plan", "rsdgc_plan_set_ratios", "rsdgc_plan_set_path", "rsdgc_plan_set_work_feed", "rsdgc_plan_forget_workspace", "rsdgc_plan_destroy", "rsdgc_n_layers",
    "rsdgc_total_elems", "rsdgc_layer_offset", "rsdgc_layer_elems", "rsdgc_layer_k",
    "rsdgc_out_offset", "rsdgc_out_capacity", "rsdgc_centre_offset", "rsdgc_centre_capacity",
    "rsdgc_workspace_bytes", "rsdgc_replaces_residual", "rsdgc_compress", "rsdgc_compress_static", "rsdgc_compress_momentum", "rsdgc_dynamic_ratios", "rsdgc_ratio_passes", "rsdgc_apply", "rsdgc_apply_blocks", "rsdgc_plan_blocks", "rsdgc_compress_blocks", "rsdgc_compress_blocks_momentum",
    "rsdgc_decompress_blocks", "rsdgc_nsi", "rsdgc_decompress",
    "rsdgc_last_paths", "rsdgc_last_paths_blocks", "rsdgc_profile_begin", "rsdgc_profile_end", "rsdgc_stage_name",
    "rsdgc_strerror", "rsdgc_last_hip_error",
    "rsdgc_layer_norm", "rsdgc_layer_norm_backward", "rsdgc_layer_norm_workspace_bytes",
    "rsdgc_head_loss", "rsdgc_head_loss_backward", "rsdgc_distill_loss", "rsdgc_distill_loss_backward",
    "rsdgc_head_workspace_bytes",
]
RSDGC_N_STAGES = 9
RSDGC_PATH_AUTO, RSDGC_PATH_FULL_MAP = 0, 1
RSDGC_F32, RSDGC_BF16 = 0, 1
RSDGC_MAX_TOP = 1024


class Shape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class RsdgcError(RuntimeError):
    def __init__(self, code: int, where: str):
        lib = load()
        msg = lib.rsdgc_strerror(code).decode()
        hip = lib.rsdgc_last_hip_error().decode()
        super().__init__(f"{where}: {msg} ({code})" +
                         (f" [{hip}]" if code in (RSDGC_EHIP, RSDGC_ETOOBIG) and hip else ""))
        self.code = code


_lib = None


def load() -> ctypes.CDLL:
    """Load librsdgc.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2312_17530_amd.build` "
            "(or __graft_entry__.build()); there is no fallback implementation")
    # PyTorch ships its own HIP runtime; it has to be in the process before this library
    # is loaded so that both resolve the same runtime (device pointers and streams are
    # only meaningful inside the runtime that created them).
    import torch  # noqa: F401
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
    lib.rsdgc_plan.argtypes = [ctypes.POINTER(Shape), i32, i32, ctypes.POINTER(i32), f64,
                               ctypes.POINTER(f64), ctypes.POINTER(vp)]
    lib.rsdgc_plan.restype = ctypes.c_int
    lib.rsdgc_plan_set_ratios.argtypes = [vp, ctypes.POINTER(f64)]
    lib.rsdgc_plan_set_ratios.restype = ctypes.c_int
    lib.rsdgc_plan_set_path.argtypes = [vp, i32]
    lib.rsdgc_plan_set_path.restype = ctypes.c_int
    lib.rsdgc_plan_set_work_feed.argtypes = [vp, i32]
    lib.rsdgc_plan_set_work_feed.restype = ctypes.c_int
    lib.rsdgc_plan_forget_workspace.argtypes = [vp]
    lib.rsdgc_plan_forget_workspace.restype = ctypes.c_int
    lib.rsdgc_plan_destroy.argtypes = [vp]
    lib.rsdgc_plan_destroy.restype = None
    lib.rsdgc_n_layers.argtypes = [vp]
    lib.rsdgc_n_layers.restype = i32
    for name in ["rsdgc_total_elems", "rsdgc_out_capacity", "rsdgc_centre_capacity"]:
        getattr(lib, name).argtypes = [vp]
        getattr(lib, name).restype = i64
    for name in ["rsdgc_layer_offset", "rsdgc_layer_elems", "rsdgc_layer_k", "rsdgc_out_offset",
                 "rsdgc_centre_offset"]:
        getattr(lib, name).argtypes = [vp, i32]
        getattr(lib, name).restype = i64
    lib.rsdgc_workspace_bytes.argtypes = [vp]
    lib.rsdgc_workspace_bytes.restype = ctypes.c_size_t
    lib.rsdgc_replaces_residual.argtypes = [vp]
    lib.rsdgc_replaces_residual.restype = i32
    lib.rsdgc_compress.argtypes = [vp] * 11
    lib.rsdgc_compress.restype = ctypes.c_int
    lib.rsdgc_compress_static.argtypes = [vp] * 10
    lib.rsdgc_compress_static.restype = ctypes.c_int
    lib.rsdgc_compress_momentum.argtypes = [vp, vp, vp, vp, ctypes.c_float] + [vp] * 9
    lib.rsdgc_compress_momentum.restype = ctypes.c_int
    lib.rsdgc_dynamic_ratios.argtypes = [vp, vp, f64, ctypes.POINTER(f64), vp, vp]
    lib.rsdgc_dynamic_ratios.restype = ctypes.c_int
    lib.rsdgc_ratio_passes.argtypes = [vp]
    lib.rsdgc_ratio_passes.restype = i32
    lib.rsdgc_apply.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), vp,
                                ctypes.c_float, vp, vp]
    lib.rsdgc_apply.restype = ctypes.c_int
    lib.rsdgc_apply_blocks.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), vp,
                                ctypes.c_float, vp, vp]
    lib.rsdgc_apply_blocks.restype = ctypes.c_int
    lib.rsdgc_plan_blocks.argtypes = lib.rsdgc_plan.argtypes
    lib.rsdgc_plan_blocks.restype = ctypes.c_int
    lib.rsdgc_compress_blocks.argtypes = [vp] * 9
    lib.rsdgc_compress_blocks.restype = ctypes.c_int
    lib.rsdgc_compress_blocks_momentum.argtypes = [vp, vp, vp, vp, ctypes.c_float] + [vp] * 7
    lib.rsdgc_compress_blocks_momentum.restype = ctypes.c_int
    lib.rsdgc_decompress_blocks.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int, vp, vp]
    lib.rsdgc_decompress_blocks.restype = ctypes.c_int
    lib.rsdgc_nsi.argtypes = [vp] * 6
    lib.rsdgc_nsi.restype = ctypes.c_int
    lib.rsdgc_decompress.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int, vp, vp]
    lib.rsdgc_decompress.restype = ctypes.c_int
    lib.rsdgc_last_paths.argtypes = [vp, vp, ctypes.POINTER(i32), vp]
    lib.rsdgc_last_paths.restype = ctypes.c_int
    lib.rsdgc_last_paths_blocks.argtypes = [vp, vp, ctypes.POINTER(i32), vp]
    lib.rsdgc_last_paths_blocks.restype = ctypes.c_int
    lib.rsdgc_profile_begin.argtypes = [vp, i32]
    lib.rsdgc_profile_begin.restype = ctypes.c_int
    lib.rsdgc_profile_end.argtypes = [vp, ctypes.POINTER(f64), ctypes.POINTER(i32)]
    lib.rsdgc_profile_end.restype = ctypes.c_int
    lib.rsdgc_stage_name.argtypes = [i32]
    lib.rsdgc_stage_name.restype = ctypes.c_char_p
    lib.rsdgc_strerror.argtypes = [ctypes.c_int]
    lib.rsdgc_strerror.restype = ctypes.c_char_p
    lib.rsdgc_last_hip_error.argtypes = []
    lib.rsdgc_last_hip_error.restype = ctypes.c_char_p
    size, flag = ctypes.c_size_t, ctypes.c_int
    lib.rsdgc_layer_norm.argtypes = [i32, i64, i64, vp, i64, vp, vp, f64, vp, i64, vp, vp, vp]
    lib.rsdgc_layer_norm_backward.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, flag, vp, vp]
    lib.rsdgc_layer_norm_workspace_bytes.argtypes = [i64, i64]
    head = [i32, i64, i64, i64, vp, i64, vp, i64]
    lib.rsdgc_head_loss.argtypes = head + [vp, vp, vp, vp, vp]
    lib.rsdgc_head_loss_backward.argtypes = head + [vp, vp, vp, vp, i64, vp, flag, vp, vp]
    lib.rsdgc_distill_loss.argtypes = head + [i32, vp, vp, f64, vp, vp, vp, vp]
    lib.rsdgc_distill_loss_backward.argtypes = head + [i32, vp, vp, f64, vp, vp, vp, i64, vp, flag, vp, vp]
    lib.rsdgc_head_workspace_bytes.argtypes = [i32, i64, i64, i64, i32, flag]
    for name in ["rsdgc_layer_norm", "rsdgc_layer_norm_backward", "rsdgc_head_loss", "rsdgc_head_loss_backward",
                 "rsdgc_distill_loss", "rsdgc_distill_loss_backward"]:
        getattr(lib, name).restype = ctypes.c_int
    for name in ["rsdgc_layer_norm_workspace_bytes", "rsdgc_head_workspace_bytes"]:
        getattr(lib, name).restype = size
    _lib = lib
    return lib


def _check(code: int, where: str) -> None:
    if code != RSDGC_OK:
        raise RsdgcError(code, where)


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a torch tensor, None for None."""
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    h = stream if isinstance(stream, int) else stream.cuda_stream
    return h or None


class Plan:
    """Owner of one rsdgc_plan_t (host object)."""

    def __init__(self, handle: int):
        self._h = ctypes.c_void_p(handle)

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:        # at interpreter shutdown the module may already be gone
            _lib.rsdgc_plan_destroy(h)

    @property
    def handle(self):
        return self._h

    @property
    def n_layers(self) -> int:
        return load().rsdgc_n_layers(self._h)

    @property
    def total_elems(self) -> int:
        return load().rsdgc_total_elems(self._h)

    @property
    def out_capacity(self) -> int:
        return load().rsdgc_out_capacity(self._h)

    @property
    def centre_capacity(self) -> int:
        return load().rsdgc_centre_capacity(self._h)

    @property
    def workspace_bytes(self) -> int:
        return load().rsdgc_workspace_bytes(self._h)

    @property
    def replaces_residual(self) -> bool:
        """Whether an update in place stores v as it is formed (else g and r are streamed once more)."""
        return load().rsdgc_replaces_residual(self._h) == 1

    def layer_offset(self, l: int) -> int:
        return load().rsdgc_layer_offset(self._h, l)

    def layer_elems(self, l: int) -> int:
        return load().rsdgc_layer_elems(self._h, l)

    def layer_k(self, l: int) -> int:
        return load().rsdgc_layer_k(self._h, l)

    def out_offset(self, l: int) -> int:
        return load().rsdgc_out_offset(self._h, l)

    def centre_offset(self, l: int) -> int:
        return load().rsdgc_centre_offset(self._h, l)


def rsdgc_plan(shapes: Sequence[Tuple[int, int]], p: int, alpha: float,
               keep_ratio: Sequence[float], p_per_layer: Optional[Sequence[int]] = None,
               blocks: bool = False) -> Plan:
    """blocks=True: rsdgc_plan_blocks (non-overlapping p x p neighbourhoods)."""
    lib = load()
    n = len(shapes)
    if len(keep_ratio) != n or (p_per_layer is not None and len(p_per_layer) != n):
        raise RsdgcError(RSDGC_EINVAL, "rsdgc_plan")
    arr = (Shape * max(n, 1))(*[Shape(int(r), int(c)) for r, c in shapes])
    ratios = (ctypes.c_double * max(len(keep_ratio), 1))(*[float(x) for x in keep_ratio])
    pp = None
    if p_per_layer is not None:
        pp = (ctypes.c_int32 * max(n, 1))(*[int(x) for x in p_per_layer])
    out = ctypes.c_void_p()
    fn = lib.rsdgc_plan_blocks if blocks else lib.rsdgc_plan
    _check(fn(arr, n, int(p), pp, float(alpha), ratios, ctypes.byref(out)),
           "rsdgc_plan_blocks" if blocks else "rsdgc_plan")
    return Plan(out.value)


def rsdgc_plan_blocks(shapes, p: int, alpha: float, keep_ratio, p_per_layer=None) -> Plan:
    return rsdgc_plan(shapes, p, alpha, keep_ratio, p_per_layer, blocks=True)


def rsdgc_compress_blocks(plan: Plan, grad, residual, residual_out, out_block_idx, out_val, out_counts,
                          workspace, stream=None) -> None:
    _check(load().rsdgc_compress_blocks(plan.handle, _ptr(grad), _ptr(residual), _ptr(residual_out),
                                        _ptr(out_block_idx), _ptr(out_val), _ptr(out_counts),
                                        _ptr(workspace), _stream(stream)), "rsdgc_compress_blocks")


def rsdgc_compress_blocks_momentum(plan: Plan, grad, momentum, momentum_out, m: float, residual, residual_out,
                                   out_block_idx, out_val, out_counts, workspace, stream=None) -> None:
    _check(load().rsdgc_compress_blocks_momentum(plan.handle, _ptr(grad), _ptr(momentum), _ptr(momentum_out),
                                                 float(m), _ptr(residual), _ptr(residual_out),
                                                 _ptr(out_block_idx), _ptr(out_val), _ptr(out_counts),
                                                 _ptr(workspace), _stream(stream)),
           "rsdgc_compress_blocks_momentum")


def rsdgc_decompress_blocks(plan: Plan, block_idx, val, counts, dense, accumulate: bool, workspace,
                            stream=None) -> None:
    _check(load().rsdgc_decompress_blocks(plan.handle, _ptr(block_idx), _ptr(val), _ptr(counts), _ptr(dense),
                                          1 if accumulate else 0, _ptr(workspace), _stream(stream)),
           "rsdgc_decompress_blocks")


def rsdgc_plan_set_ratios(plan: Plan, keep_ratio: Sequence[float]) -> None:
    if len(keep_ratio) != plan.n_layers:
        raise RsdgcError(RSDGC_EINVAL, "rsdgc_plan_set_ratios")
    ratios = (ctypes.c_double * len(keep_ratio))(*[float(x) for x in keep_ratio])
    _check(load().rsdgc_plan_set_ratios(plan.handle, ratios), "rsdgc_plan_set_ratios")


FEED_AUTO, FEED_OFF, FEED_ON = 0, 1, 2


def rsdgc_plan_forget_workspace(plan: "Plan") -> None:
    _check(load().rsdgc_plan_forget_workspace(plan.handle), "rsdgc_plan_forget_workspace")


def rsdgc_plan_set_work_feed(plan: "Plan", mode: int) -> None:
    _check(load().rsdgc_plan_set_work_feed(plan.handle, int(mode)), "rsdgc_plan_set_work_feed")


def rsdgc_plan_set_path(plan: Plan, path: int) -> None:
    _check(load().rsdgc_plan_set_path(plan.handle, int(path)), "rsdgc_plan_set_path")


def rsdgc_compress(plan: Plan, grad, residual, residual_out, out_idx, out_val, out_counts, workspace,
                   out_centre_idx=None, out_centre_counts=None, stream=None) -> None:
    """residual_out is a second arena, or the same tensor as residual for an update in place."""
    _check(load().rsdgc_compress(plan.handle, _ptr(grad), _ptr(residual), _ptr(residual_out), _ptr(out_idx),
                                 _ptr(out_val), _ptr(out_counts), _ptr(out_centre_idx),
                                 _ptr(out_centre_counts), _ptr(workspace), _stream(stream)),
           "rsdgc_compress")


def rsdgc_compress_static(plan: Plan, grad, residual, residual_out, out_idx, out_val, out_counts,
                          out_centre_idx=None, out_centre_counts=None, stream=None) -> None:
    """rsdgc_compress with the library's built-in workspace (no device allocation)."""
    _check(load().rsdgc_compress_static(plan.handle, _ptr(grad), _ptr(residual), _ptr(residual_out),
                                        _ptr(out_idx), _ptr(out_val), _ptr(out_counts), _ptr(out_centre_idx),
                                        _ptr(out_centre_counts), _stream(stream)), "rsdgc_compress_static")


def rsdgc_compress_momentum(plan: Plan, grad, momentum, momentum_out, m: float, residual, residual_out,
                            out_idx, out_val, out_counts, workspace, out_centre_idx=None,
                            out_centre_counts=None, stream=None) -> None:
    """Eq. 12 in full; the five arenas must not overlap."""
    _check(load().rsdgc_compress_momentum(plan.handle, _ptr(grad), _ptr(momentum), _ptr(momentum_out),
                                          float(m), _ptr(residual), _ptr(residual_out), _ptr(out_idx),
                                          _ptr(out_val), _ptr(out_counts), _ptr(out_centre_idx),
                                          _ptr(out_centre_counts), _ptr(workspace), _stream(stream)),
           "rsdgc_compress_momentum")


def rsdgc_dynamic_ratios(plan: Plan, weights, global_ratio: float, workspace, stream=None) -> List[float]:
    """Eqs. 3-5: per-layer keep ratios from the weights arena (waits for the GPU)."""
    out = (ctypes.c_double * plan.n_layers)()
    _check(load().rsdgc_dynamic_ratios(plan.handle, _ptr(weights), float(global_ratio), out,
                                       _ptr(workspace), _stream(stream)), "rsdgc_dynamic_ratios")
    return [float(x) for x in out]


def rsdgc_ratio_passes(plan: Plan) -> int:
    """Streaming passes of the last rsdgc_dynamic_ratios call: 1, or 4 or 5 on the general path."""
    return load().rsdgc_ratio_passes(plan.handle)


def rsdgc_apply(plan: Plan, messages, weights, eta: float, workspace, stream=None) -> None:
    """Eq. 12, third line: weights -= eta * (sum of the messages, in order).
    messages: sequence of (idx, val, counts) device tensors as written by rsdgc_compress."""
    n = len(messages)
    arr = ctypes.c_void_p * max(n, 1)
    idx = arr(*[_ptr(m[0]) for m in messages])
    val = arr(*[_ptr(m[1]) for m in messages])
    cnt = arr(*[_ptr(m[2]) for m in messages])
    _check(load().rsdgc_apply(plan.handle, n, idx, val, cnt, _ptr(weights), float(eta), _ptr(workspace),
                              _stream(stream)), "rsdgc_apply")


def rsdgc_apply_blocks(plan: Plan, messages, weights, eta: float, workspace, stream=None) -> None:
    """rsdgc_apply for a block plan.  messages: sequence of (block_idx, val, counts) device
    tensors as written by rsdgc_compress_blocks."""
    n = len(messages)
    arr = ctypes.c_void_p * max(n, 1)
    idx = arr(*[_ptr(m[0]) for m in messages])
    val = arr(*[_ptr(m[1]) for m in messages])
    cnt = arr(*[_ptr(m[2]) for m in messages])
    _check(load().rsdgc_apply_blocks(plan.handle, n, idx, val, cnt, _ptr(weights), float(eta), _ptr(workspace),
                                     _stream(stream)), "rsdgc_apply_blocks")


def rsdgc_nsi(plan: Plan, grad, residual, nsi_out, workspace, stream=None) -> None:
    _check(load().rsdgc_nsi(plan.handle, _ptr(grad), _ptr(residual), _ptr(nsi_out),
                            _ptr(workspace), _stream(stream)), "rsdgc_nsi")


def rsdgc_decompress(plan: Plan, idx, val, counts, dense, accumulate: bool, workspace,
                     stream=None) -> None:
    _check(load().rsdgc_decompress(plan.handle, _ptr(idx), _ptr(val), _ptr(counts), _ptr(dense),
                                   1 if accumulate else 0, _ptr(workspace), _stream(stream)),
           "rsdgc_decompress")


def rsdgc_profile_begin(plan: Plan, max_calls: int) -> None:
    _check(load().rsdgc_profile_begin(plan.handle, int(max_calls)), "rsdgc_profile_begin")


def rsdgc_profile_end(plan: Plan):
    """Returns ({stage name: mean ms per call}, number of recorded calls)."""
    lib = load()
    ms = (ctypes.c_double * RSDGC_N_STAGES)()
    n = ctypes.c_int32(0)
    _check(lib.rsdgc_profile_end(plan.handle, ms, ctypes.byref(n)), "rsdgc_profile_end")
    return {lib.rsdgc_stage_name(i).decode(): ms[i] for i in range(RSDGC_N_STAGES)}, n.value


def rsdgc_last_paths(plan: Plan, workspace, stream=None):
    """Ranking path per layer of the last compress call (0 candidates above a sampled bound, 3 above a predicted
    one, 1 full map, 2 none)."""
    out = (ctypes.c_int32 * plan.n_layers)()
    _check(load().rsdgc_last_paths(plan.handle, _ptr(workspace), out, _stream(stream)),
           "rsdgc_last_paths")
    return list(out)


def rsdgc_last_paths_blocks(plan: Plan, workspace, stream=None):
    """The same of a block plan's grids in the last rsdgc_compress_blocks(_momentum) call."""
    out = (ctypes.c_int32 * plan.n_layers)()
    _check(load().rsdgc_last_paths_blocks(plan.handle, _ptr(workspace), out, _stream(stream)),
           "rsdgc_last_paths_blocks")
    return list(out)


# ------------------------------------------------------ training operators
# These calls can be as short as a launch (a few microseconds), so what they check is kept lean.
_torch = None
_CODES: dict = {}          # torch dtype -> RSDGC_F32 / RSDGC_BF16


def _training():
    """The library; torch and the dtype codes are at hand afterwards."""
    global _torch
    if _torch is None:
        import torch
        _CODES.update({torch.float32: RSDGC_F32, torch.bfloat16: RSDGC_BF16})
        _torch = torch
    return _lib if _lib is not None else load()


def _dtype(dtype) -> int:
    """RSDGC_F32 or RSDGC_BF16 of a torch dtype."""
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"float32 or bfloat16 is needed, got {dtype}")
    return code


def _need(ok: bool, where: str) -> None:
    """The library sees addresses only: what they hold is checked here."""
    if not ok:
        raise RsdgcError(RSDGC_EINVAL, where)


def _stream_on(t, stream) -> Optional[int]:
    """The stream given, or the current one of t's device (t's device has to be the current one, as for every call)."""
    if stream is None:
        return _torch._C._cuda_getCurrentRawStream(t.get_device()) or None
    return _stream(stream)


def _rows(t, dtype, shape, dev: int, where: str):
    """(address, stride between rows) of a matrix of `shape` on device `dev` whose rows are without gaps."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _need(False, where)
    rows, cols = shape
    down, along = t.stride()
    if along != 1 and cols > 1:
        _need(False, where)
    # with a single row (or none) the stride says nothing
    return t.data_ptr(), (down if rows > 1 else cols)


def _flat(t, n: int, dtype, dev: int, where: str) -> Optional[int]:
    """Address of n elements on device `dev` without gaps."""
    if t is None:
        return None
    if t.numel() != n or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _need(False, where)
    return t.data_ptr()


def _bytes(workspace, need: int, dev: int, where: str) -> Optional[int]:
    _need(workspace is not None and workspace.is_contiguous() and workspace.get_device() == dev
          and workspace.numel() * workspace.element_size() >= need, where)
    return workspace.data_ptr()


def _matrix(x, where: str):
    """(library, code, shape, device) of the operand that the others follow; no kernel can read another device's memory."""
    lib = _training()
    shape, dev = x.shape, x.get_device()
    _need(len(shape) == 2 and dev >= 0, where)
    return lib, _dtype(x.dtype), shape, dev


def rsdgc_layer_norm(x, gamma, beta, eps: float, y, mean=None, rstd=None, stream=None) -> None:
    """y = (x - mean) * rstd * gamma + beta over the rows of x; mean and rstd are kept for the backward pass if given."""
    where = "rsdgc_layer_norm"
    lib, code, shape, dev = _matrix(x, where)
    rows, cols = shape
    px, ldx = _rows(x, x.dtype, shape, dev, where)
    py, ldy = _rows(y, x.dtype, shape, dev, where)
    f32 = _torch.float32
    _check(lib.rsdgc_layer_norm(code, rows, cols, px, ldx, _flat(gamma, cols, f32, dev, where), _flat(beta, cols, f32, dev, where), eps,
                                py, ldy, _flat(mean, rows, f32, dev, where), _flat(rstd, rows, f32, dev, where), _stream_on(x, stream)),
           where)


def rsdgc_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    n = load().rsdgc_layer_norm_workspace_bytes(rows, cols)
    _need(n > 0, "rsdgc_layer_norm_workspace_bytes")
    return n


def rsdgc_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, accumulate: bool, workspace, stream=None) -> None:
    """dx, and dgamma / dbeta (float32, e.g. layers of the gradient arena; None: not wanted) of rsdgc_layer_norm."""
    where = "rsdgc_layer_norm_backward"
    lib, code, shape, dev = _matrix(x, where)
    rows, cols = shape
    px, ldx = _rows(x, x.dtype, shape, dev, where)
    pdy, lddy = _rows(dy, x.dtype, shape, dev, where)
    pdx, lddx = _rows(dx, x.dtype, shape, dev, where)
    _need(mean is not None and rstd is not None, where)
    ws = None
    if dgamma is not None or dbeta is not None:
        ws = _bytes(workspace, lib.rsdgc_layer_norm_workspace_bytes(rows, cols), dev, where)
    f32 = _torch.float32
    _check(lib.rsdgc_layer_norm_backward(code, rows, cols, pdy, lddy, px, ldx, _flat(gamma, cols, f32, dev, where),
                                         _flat(mean, rows, f32, dev, where), _flat(rstd, rows, f32, dev, where), pdx, lddx,
                                         _flat(dgamma, cols, f32, dev, where), _flat(dbeta, cols, f32, dev, where),
                                         1 if accumulate else 0, ws, _stream_on(x, stream)), where)


def rsdgc_head_workspace_bytes(dtype, rows: int, hidden: int, vocab: int, top: int = 0, backward: bool = True) -> int:
    """top: 0 for cross entropy, else the teacher's kept logits per row."""
    n = _training().rsdgc_head_workspace_bytes(_dtype(dtype), rows, hidden, vocab, top, 1 if backward else 0)
    _need(n > 0, "rsdgc_head_workspace_bytes")
    return n


def _head(x, w, top: int, workspace, backward: bool, where: str):
    """The library, the arguments that the head's calls begin with, and the workspace's address."""
    lib, code, shape, dev = _matrix(x, where)
    rows, hidden = shape
    _need(w.dim() == 2 and w.shape[1] == hidden, where)
    px, ldx = _rows(x, x.dtype, shape, dev, where)
    pw, ldw = _rows(w, x.dtype, w.shape, dev, where)
    vocab = w.shape[0]
    need = lib.rsdgc_head_workspace_bytes(code, rows, hidden, vocab, top, 1 if backward else 0)
    _need(need > 0, where)
    return lib, (code, rows, hidden, vocab, px, ldx, pw, ldw), _bytes(workspace, need, dev, where)


def _head_gradients(x, w, lse, row_grad, dx, dw, accumulate: bool, where: str):
    (rows, hidden), dev = x.shape, x.get_device()
    f32 = _torch.float32
    pdx, lddx = _rows(dx, x.dtype, x.shape, dev, where)
    _need(lse is not None and row_grad is not None and dw is not None, where)
    return (_flat(lse, rows, f32, dev, where), _flat(row_grad, rows, f32, dev, where), pdx, lddx, _flat(dw, w.shape[0] * hidden, f32, dev, where),
            1 if accumulate else 0)


def rsdgc_head_loss(x, w, target, loss, lse, workspace, stream=None) -> None:
    """Softmax cross entropy of the logits x w^T against target (int32; outside the vocabulary: no answer), per row."""
    where = "rsdgc_head_loss"
    lib, args, ws = _head(x, w, 0, workspace, False, where)
    n, f32, dev = x.shape[0], _torch.float32, x.get_device()
    _check(lib.rsdgc_head_loss(*args, _flat(target, n, _torch.int32, dev, where), _flat(loss, n, f32, dev, where), _flat(lse, n, f32, dev, where),
                               ws, _stream_on(x, stream)), where)


def rsdgc_head_loss_backward(x, w, target, lse, row_grad, dx, dw, accumulate: bool, workspace, stream=None) -> None:
    """dx, and dw (float32, vocabulary x width without gaps, e.g. a layer of the gradient arena), of rsdgc_head_loss."""
    where = "rsdgc_head_loss_backward"
    lib, args, ws = _head(x, w, 0, workspace, True, where)
    _check(lib.rsdgc_head_loss_backward(*args, _flat(target, x.shape[0], _torch.int32, x.get_device(), where),
                                        *_head_gradients(x, w, lse, row_grad, dx, dw, accumulate, where), ws,
                                        _stream_on(x, stream)), where)


def _teacher(x, top_idx, top_logit, where: str):
    _training()
    _need(top_idx.dim() == 2 and top_idx.shape[0] == x.shape[0] and top_logit.shape == top_idx.shape
          and 1 <= top_idx.shape[1] <= RSDGC_MAX_TOP, where)
    n, dev = top_idx.numel(), x.get_device()
    return top_idx.shape[1], _flat(top_idx, n, _torch.int32, dev, where), _flat(top_logit, n, _torch.float32, dev, where)


def rsdgc_distill_loss(x, w, top_idx, top_logit, temperature: float, loss, lse, workspace, stream=None) -> None:
    """Distillation from a teacher's kept logits (top_idx int32, top_logit float32, both [rows, top]), per row."""
    where = "rsdgc_distill_loss"
    top = _teacher(x, top_idx, top_logit, where)
    lib, args, ws = _head(x, w, top[0], workspace, False, where)
    n, f32, dev = x.shape[0], _torch.float32, x.get_device()
    _check(lib.rsdgc_distill_loss(*args, *top, temperature, _flat(loss, n, f32, dev, where), _flat(lse, n, f32, dev, where), ws,
                                  _stream_on(x, stream)), where)


def rsdgc_distill_loss_backward(x, w, top_idx, top_logit, temperature: float, lse, row_grad, dx, dw, accumulate: bool, workspace,
                                stream=None) -> None:
    """dx and dw of rsdgc_distill_loss, as rsdgc_head_loss_backward."""
    where = "rsdgc_distill_loss_backward"
    top = _teacher(x, top_idx, top_logit, where)
    lib, args, ws = _head(x, w, top[0], workspace, True, where)
    _check(lib.rsdgc_distill_loss_backward(*args, *top, temperature, *_head_gradients(x, w, lse, row_grad, dx, dw, accumulate, where),
                                           ws, _stream_on(x, stream)), where)
