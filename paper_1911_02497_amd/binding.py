"""ctypes binding of libcondensa.so: same names as the C entry points, marshalling only.

torch is used for device memory and the current stream; no arithmetic happens here.
"""
from __future__ import annotations

import array
import ctypes
import functools
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# CONDENSA_LIBRARY names another build of the same library (same C ABI), e.g. one compiled elsewhere.
_LIB_PATH = os.environ.get("CONDENSA_LIBRARY") or os.path.join(_HERE, "libcondensa.so")

SCOPE_GLOBAL, SCOPE_PER_TENSOR = 0, 1
OP_PRUNE, OP_FILTER_PRUNE, OP_BLOCK_PRUNE, OP_QUANTIZE, OP_LC_STEP, OP_COUNT_NONZERO, OP_LC_SGD_STEP = range(7)
OPT_SELECT_PATH, OPT_SAMPLE_LOG2, OPT_WINDOW_MARGIN, OPT_CAND_SHIFT, OPT_PROFILE, OPT_APPLY_THREADS, OPT_FUSED_SWEEP = range(7)
WINDOW_MARGIN_DEFAULT = 80          # CONDENSA_OPT_WINDOW_MARGIN as the library starts with
PHASES = ("sample", "sweep", "resolve", "apply", "aggregate")
MAX_DENSITIES = 16

SELECT_FIELDS = ("n", "k", "n_gt", "n_tie_kept", "n_tie", "threshold_key", "tie_end", "path")


class CondensaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"condensa status {code}: {msg}")
        self.code = code


class Config(ctypes.Structure):
    """condensa_config: the tuning / test knobs of one call."""
    _fields_ = [("select_path", ctypes.c_int32), ("sample_log2", ctypes.c_int32), ("window_margin", ctypes.c_int32),
                ("cand_shift", ctypes.c_int32), ("profile", ctypes.c_int32), ("apply_threads", ctypes.c_int32),
                ("fused_sweep", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Tensor(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("shape", ctypes.c_int64 * 4), ("ndim", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("w", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "theta",
                                               "lambda_", "codes")] + [("n", ctypes.c_uint64)]


class AdamwList(ctypes.Structure):
    _fields_ = [("table_dev", ctypes.c_void_p), ("map_dev", ctypes.c_void_p), ("n_elems", ctypes.c_uint64), ("n_chunks", ctypes.c_uint64),
                ("n_tensors", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("code_type", ctypes.c_int32)]


class AdamwSettings(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("mu", ctypes.c_float), ("rounding", ctypes.c_int32), ("step", ctypes.c_int64),
                ("seed", ctypes.c_uint64), ("grad_scale_dev", ctypes.c_void_p), ("reserved", ctypes.c_int64)]


class Adapter(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("grad_a", ctypes.c_void_p), ("grad_b", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("rank", ctypes.c_int32)]


class AdapterList(ctypes.Structure):
    _fields_ = [("table_dev", ctypes.c_void_p), ("n_in", ctypes.c_int64), ("n_out", ctypes.c_int64), ("n_adapters", ctypes.c_int32),
                ("max_rank", ctypes.c_int32), ("type", ctypes.c_int32), ("flags", ctypes.c_int32)]


_PROTOTYPES = {
    "condensa_adapter_list_bytes": (ctypes.c_size_t, [ctypes.c_int]),
    "condensa_adapter_list_init": (ctypes.c_int32, [ctypes.POINTER(Adapter), ctypes.c_int, ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                                                    ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(AdapterList)]),
    "condensa_adapter_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(AdapterList), ctypes.c_int64, ctypes.c_int]),
    "condensa_adapter_project": (ctypes.c_int32, [ctypes.POINTER(AdapterList), ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                                  ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                                  ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "condensa_adapter_project_backward": (ctypes.c_int32, [ctypes.POINTER(AdapterList), ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                                           ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "condensa_adamw_list_bytes": (ctypes.c_size_t, [ctypes.POINTER(AdamwTensor), ctypes.c_int]),
    "condensa_adamw_list_init": (ctypes.c_int32, [ctypes.POINTER(AdamwTensor), ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                  ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(AdamwList)]),
    "condensa_lc_adamw_step": (ctypes.c_int32, [ctypes.POINTER(AdamwList), ctypes.POINTER(AdamwSettings), ctypes.c_void_p]),
    "condensa_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int,
                                                   ctypes.c_int, ctypes.c_int, ctypes.POINTER(Config)]),
    "condensa_config_init": (ctypes.c_int32, [ctypes.POINTER(Config)]),
    "condensa_prune_static": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                               ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                               ctypes.c_void_p, ctypes.c_void_p]),
    "condensa_prune": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                        ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_filter_prune": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_double, ctypes.c_int,
                                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                               ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_neuron_prune": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_double, ctypes.c_int,
                                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                               ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_structure_prune": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_double, ctypes.c_int,
                                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                  ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_block_prune_nd": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.POINTER(ctypes.c_int32),
                                                 ctypes.c_int, ctypes.c_double, ctypes.c_int, ctypes.c_void_p,
                                                 ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                 ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                 ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_block_prune": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                              ctypes.c_double, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_quantize": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_void_p]),
    "condensa_dequantize": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p]),
    "condensa_quantize_bf16": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_void_p]),
    "condensa_dequantize_bf16": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p]),
    "condensa_quantize_fp8": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p,
                                               ctypes.c_void_p, ctypes.c_void_p]),
    "condensa_dequantize_fp8": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p,
                                                 ctypes.c_void_p]),
    "condensa_lc_step": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_float, ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                          ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_lc_step_pq": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_float, ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_count_nonzero": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                                ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_lc_sgd_step": (ctypes.c_int32, [ctypes.POINTER(Tensor), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float, ctypes.c_float,
                                              ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.POINTER(Config)]),
    "condensa_mu_schedule": (ctypes.c_float, [ctypes.c_double, ctypes.c_double, ctypes.c_int]),
    "condensa_thin": (ctypes.c_int32, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64), ctypes.c_int, ctypes.c_void_p,
                                       ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                       ctypes.c_void_p, ctypes.c_void_p]),
    "condensa_set_option": (ctypes.c_int32, [ctypes.c_int, ctypes.c_int64]),
    "condensa_get_option": (ctypes.c_int64, [ctypes.c_int]),
    "condensa_profile_read": (ctypes.c_int32, [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                               ctypes.POINTER(ctypes.c_uint64)]),
    "condensa_profile_reset": (ctypes.c_int32, []),
    "condensa_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "condensa_last_hip_error": (ctypes.c_int, []),
    "condensa_launch_count": (ctypes.c_uint64, []),
    "condensa_version": (ctypes.c_int, []),
}


def exported_symbols() -> List[str]:
    """Names every entry point declared in include/condensa.h must be exported under."""
    return sorted(_PROTOTYPES)


_lib = None


def library() -> ctypes.CDLL:
    """Loads libcondensa.so (after torch, so both share one HIP runtime).  No fallback exists."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_1911_02497_amd.build` "
                "(there is no CPU or PyTorch fallback)")
        import torch  # noqa: F401  (brings in the HIP runtime the library binds to)
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _PROTOTYPES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(code: int) -> None:
    if code:
        lib = library()
        msg = lib.condensa_status_string(code).decode()
        if code == -7:
            msg += f" (hipError {lib.condensa_last_hip_error()})"
        raise CondensaError(code, msg)


@functools.lru_cache(None)
def _raw_stream():
    """Device index -> handle of its current stream.  torch's own function for that makes no Stream object, which is a microsecond less
    a call; it is not public, so the public way stands in where a version of torch lacks it."""
    import torch
    return getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: int(torch.cuda.current_stream(index).cuda_stream))


def _stream(stream) -> int:
    import torch
    if stream is None:
        return _raw_stream()(torch.cuda.current_device())
    return int(stream.cuda_stream)


class TensorTable(list):
    """A list of weight tensors together with its marshalled ``condensa_tensor`` array.  Passing one
    instead of a plain list to the calls below skips the per-call marshalling (it matters for models with
    many small tensors, where the Python loop costs more than the GPU work).  The tensors must keep their
    storage: a tensor that is reallocated needs a new table."""

    def __init__(self, tensors):
        super().__init__(tensors)
        self._arr = _marshal_tensors(self)
        self._total = sum(t.numel() for t in self)
        self._cache = {}

    def cached(self, key, make):
        if key not in self._cache:
            self._cache[key] = make()
        return self._cache[key]


def tensor_table(tensors) -> TensorTable:
    return tensors if isinstance(tensors, TensorTable) else TensorTable(tensors)


def _marshal_tensors(tensors):
    import torch
    arr = (Tensor * max(len(tensors), 1))()
    for i, t in enumerate(tensors):
        if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            raise TypeError("weights must be contiguous float32 device tensors")
        if t.dim() < 1 or t.dim() > 4:
            raise ValueError("weights must have 1 to 4 dimensions")
        arr[i].w = t.data_ptr() if t.numel() else None
        for d in range(t.dim()):
            arr[i].shape[d] = t.shape[d]
        arr[i].ndim = t.dim()
        arr[i].reserved = 0
    return arr


def _tensor_table(tensors):
    return tensors._arr if isinstance(tensors, TensorTable) else _marshal_tensors(tensors)


def _total(tensors) -> int:
    return tensors._total if isinstance(tensors, TensorTable) else sum(t.numel() for t in tensors)


def _cached(tensors, key, make):
    return tensors.cached(key, make) if isinstance(tensors, TensorTable) else make()


def _ptr_table(tensors: Optional[Sequence]):
    """Host array of device pointers (None entries and tensors without elements become NULL); None -> NULL table.
    The first value owns the memory that the second points to."""
    if tensors is None:
        return None, None
    arr = array.array("Q", [0 if t is None else t.data_ptr() for t in tensors] or [0])     # data_ptr of an empty tensor is 0
    return arr, ctypes.c_void_p(arr.buffer_info()[0])


def condensa_config(**fields) -> Config:
    """A condensa_config holding the process-wide defaults, with the given fields changed
    (select_path, sample_log2, window_margin, cand_shift, profile, apply_threads, fused_sweep)."""
    c = Config()
    _check(library().condensa_config_init(ctypes.byref(c)))
    for k, v in fields.items():
        if k not in {f for f, _ in Config._fields_} or k == "reserved":
            raise KeyError(k)
        setattr(c, k, int(v))
    return c


def _cfg(config):
    """None -> NULL (process-wide defaults); a dict of fields or a Config -> pointer to the struct."""
    if config is None:
        return None
    if isinstance(config, dict):
        config = condensa_config(**config)
    return ctypes.byref(config)


def _workspace(op, total, n_struct, n_tensors, n_dens, scope, device, workspace=None, config=None):
    import torch
    need = int(library().condensa_workspace_bytes(op, total, n_struct, n_tensors, n_dens, scope, _cfg(config)))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace, need


def condensa_workspace_bytes(op, total_elems, n_structures, n_tensors, n_densities, scope, config=None) -> int:
    return int(library().condensa_workspace_bytes(op, total_elems, n_structures, n_tensors, n_densities, scope,
                                                  _cfg(config)))


def condensa_set_option(option: int, value: int) -> None:
    _check(library().condensa_set_option(option, value))


def condensa_get_option(option: int) -> int:
    return int(library().condensa_get_option(option))


def condensa_launch_count() -> int:
    return int(library().condensa_launch_count())


def condensa_profile_reset() -> None:
    _check(library().condensa_profile_reset())


def condensa_profile_read() -> Dict[str, Dict[str, float]]:
    """Totals of the phase intervals recorded since the last reset: {phase: {ms, intervals}}."""
    out = {}
    for i, name in enumerate(PHASES):
        ms, n = ctypes.c_double(0.0), ctypes.c_uint64(0)
        _check(library().condensa_profile_read(i, ctypes.byref(ms), ctypes.byref(n)))
        out[name] = {"ms": ms.value, "intervals": int(n.value)}
    return out


def select_records(results) -> List[Dict[str, int]]:
    """Device int64 [m, 8] record tensor -> list of dicts (synchronises)."""
    host = results.cpu().numpy().view(np.uint64).reshape(-1, len(SELECT_FIELDS))
    return [{f: int(row[i]) for i, f in enumerate(SELECT_FIELDS)} for row in host]


def condensa_prune(tensors, densities, scope=SCOPE_GLOBAL, theta=True, theta_f16=False, mask=True,
                   in_place=False, workspace=None, stream=None, outputs=None, config=None, static=False):
    """Marshals a call of the C entry point condensa_prune.  ``theta`` / ``theta_f16`` / ``mask`` choose
    which outputs are allocated ([density][tensor] lists of device tensors); ``in_place`` passes the
    weights themselves as theta (one density only).  ``static`` calls condensa_prune_static instead (no
    workspace, GLOBAL scope).  Returns the outputs and the record tensor."""
    import torch
    lib = library()
    dev = tensors[0].device if tensors else torch.device("cuda")
    nt, J = len(tensors), len(densities)
    tab = _tensor_table(tensors)
    dens = (ctypes.c_double * max(J, 1))(*[float(d) for d in densities])
    total = _total(tensors)

    outputs = (outputs or {}).get("_buffers", {})    # ``outputs``: an earlier call's result, whose tensors are reused

    def outs(flag, dtype, name):
        if not flag:
            return None
        if outputs.get(name) is not None:
            return outputs[name]
        return [[torch.empty(t.shape, dtype=dtype, device=dev) for t in tensors] for _ in range(J)]

    th = [list(tensors)] if (theta and in_place) else outs(theta, torch.float32, "theta")
    th16 = outs(theta_f16, torch.int16, "theta_f16")
    mk = outs(mask, torch.uint8, "mask")
    flat = lambda x: None if x is None else [t for row in x for t in row]  # noqa: E731
    k1, p1 = _ptr_table(flat(th))
    k2, p2 = _ptr_table(flat(th16))
    k3, p3 = _ptr_table(flat(mk))
    n_rec = J * (nt if scope == SCOPE_PER_TENSOR else 1)
    results = outputs.get("results")
    if results is None:
        results = torch.zeros((max(n_rec, 1), len(SELECT_FIELDS)), dtype=torch.int64, device=dev)
    if static:
        if scope != SCOPE_GLOBAL or config is not None or workspace is not None:
            raise ValueError("condensa_prune_static: GLOBAL scope, no workspace, built-in settings")
        ws = None
        _check(lib.condensa_prune_static(tab, nt, dens, J, p1, p2, p3, results.data_ptr(), _stream(stream)))
    else:
        ws, need = _workspace(OP_PRUNE, total, 0, nt, J, scope, dev, workspace, config)
        _check(lib.condensa_prune(tab, nt, dens, J, scope, p1, p2, p3, results.data_ptr(), ws.data_ptr(), ws.numel(),
                                  _stream(stream), _cfg(config)))
    return {"theta": th, "theta_f16": th16, "mask": mk, "results": results[:n_rec], "workspace": ws,
            "_keep": (k1, k2, k3),
            "_buffers": {"theta": None if in_place else th, "theta_f16": th16, "mask": mk, "results": results}}


def _structure_call(fn_name, op, tensors, n_struct, density, scope, theta, mask, extra_args, workspace, stream,
                    outputs=None, config=None, fill_keep_idx=False):
    import torch
    lib = library()
    dev = tensors[0].device if tensors else torch.device("cuda")
    nt = len(tensors)
    tab = _tensor_table(tensors)
    total = _total(tensors)
    o = (outputs or {}).get("_buffers", {})      # ``outputs``: an earlier call's result, whose tensors are reused
    F = max(n_struct, 1)
    n_rec = nt if scope == SCOPE_PER_TENSOR else 1

    def reuse(name, make):
        return o[name] if o.get(name) is not None else make()

    th = reuse("theta", lambda: [torch.empty_like(t) for t in tensors]) if theta else None
    mk = reuse("mask", lambda: [torch.empty(t.shape, dtype=torch.uint8, device=dev) for t in tensors]) if mask else None
    k1, p1, k2, p2 = reuse("_tables", lambda: _ptr_table(th) + _ptr_table(mk))
    sumsq = reuse("sumsq", lambda: torch.empty(F, dtype=torch.float64, device=dev))
    norms = reuse("norms", lambda: torch.empty(F, dtype=torch.float32, device=dev))
    keep_idx = reuse("keep_idx", lambda: torch.empty(F, dtype=torch.int32, device=dev))
    if fill_keep_idx:                       # the library writes the first k entries only; on request the rest reads -1
        with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
            keep_idx.fill_(-1)
    smask = reuse("structure_mask", lambda: torch.empty(F, dtype=torch.uint8, device=dev))
    results = reuse("results", lambda: torch.zeros((max(n_rec, 1), len(SELECT_FIELDS)), dtype=torch.int64, device=dev))
    ws, need = _workspace(op, total, n_struct, nt, 1, scope, dev, workspace, config)
    args = [tab, nt] + extra_args + [float(density), scope, p1, p2, sumsq.data_ptr(), norms.data_ptr(),
                                     keep_idx.data_ptr(), smask.data_ptr(), results.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _stream(stream), _cfg(config)]
    _check(getattr(lib, fn_name)(*args))
    return {"theta": th, "mask": mk, "sumsq": sumsq[:n_struct], "norms": norms[:n_struct],
            "keep_idx": keep_idx[:n_struct], "structure_mask": smask[:n_struct], "results": results[:n_rec],
            "workspace": ws, "_keep": (k1, k2),
            "_buffers": {"theta": th, "mask": mk, "sumsq": sumsq, "norms": norms, "keep_idx": keep_idx,
                         "structure_mask": smask, "results": results, "_tables": (k1, p1, k2, p2)}}


def condensa_filter_prune(tensors, density, scope=SCOPE_GLOBAL, theta=True, mask=True, workspace=None, stream=None,
                          outputs=None, **kw):
    n_struct = _cached(tensors, "rows", lambda: sum(t.shape[0] if t.numel() else 0 for t in tensors))
    return _structure_call("condensa_filter_prune", OP_FILTER_PRUNE, tensors, n_struct, density, scope, theta, mask,
                           [], workspace, stream, outputs, **kw)


def condensa_block_prune(tensors, block_h, block_w, density, scope=SCOPE_GLOBAL, theta=True, mask=True,
                         workspace=None, stream=None, outputs=None, **kw):
    n_struct = _cached(tensors, ("blocks", block_h, block_w),
                       lambda: sum((t.shape[0] // block_h) * (t.shape[1] // block_w) for t in tensors if t.dim() == 2))
    return _structure_call("condensa_block_prune", OP_BLOCK_PRUNE, tensors, n_struct, density, scope, theta, mask,
                           [int(block_h), int(block_w)], workspace, stream, outputs, **kw)


def condensa_neuron_prune(tensors, density, scope=SCOPE_GLOBAL, theta=True, mask=True, workspace=None, stream=None,
                          outputs=None, **kw):
    n_struct = _cached(tensors, "rows", lambda: sum(t.shape[0] if t.numel() else 0 for t in tensors))
    return _structure_call("condensa_neuron_prune", OP_FILTER_PRUNE, tensors, n_struct, density, scope, theta, mask,
                           [], workspace, stream, outputs, **kw)


def condensa_structure_prune(tensors, density, scope=SCOPE_GLOBAL, theta=True, mask=True, workspace=None, stream=None,
                             outputs=None, **kw):
    n_struct = _cached(tensors, "rows", lambda: sum(t.shape[0] if t.numel() else 0 for t in tensors))
    return _structure_call("condensa_structure_prune", OP_FILTER_PRUNE, tensors, n_struct, density, scope, theta, mask,
                           [], workspace, stream, outputs, **kw)


def condensa_block_prune_nd(tensors, block_shape, density, scope=SCOPE_GLOBAL, theta=True, mask=True,
                            workspace=None, stream=None, outputs=None, **kw):
    nd = len(block_shape)
    blk = (ctypes.c_int32 * max(nd, 1))(*[int(b) for b in block_shape])
    n_struct = 0
    for t in tensors:
        if t.dim() == nd and t.numel():
            c = 1
            for d, b in zip(t.shape, block_shape):
                c *= -(-d // max(int(b), 1))
            n_struct += c
    return _structure_call("condensa_block_prune_nd", OP_BLOCK_PRUNE, tensors, n_struct, density, scope, theta, mask,
                           [blk, nd], workspace, stream, outputs, **kw)


def _quantize(fn_name, x, want_q, want_dq, stream):
    import torch
    q = torch.empty(x.shape, dtype=torch.int16, device=x.device) if want_q else None
    dq = torch.empty_like(x) if want_dq else None
    _check(getattr(library(), fn_name)(x.data_ptr() if x.numel() else None, x.numel(),
                                       q.data_ptr() if q is not None else None,
                                       dq.data_ptr() if dq is not None else None, _stream(stream)))
    return q, dq


def _dequantize(fn_name, q, stream):
    import torch
    dq = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check(getattr(library(), fn_name)(q.data_ptr() if q.numel() else None, q.numel(), dq.data_ptr(), _stream(stream)))
    return dq


def condensa_quantize(x, want_q=True, want_dq=True, stream=None):
    """binary16 codes (int16 views of the bits) and / or their exact widening."""
    return _quantize("condensa_quantize", x, want_q, want_dq, stream)


def condensa_dequantize(q, stream=None):
    return _dequantize("condensa_dequantize", q, stream)


def condensa_quantize_bf16(x, want_q=True, want_dq=True, stream=None):
    """bfloat16 codes (int16 views of the bits) and / or their exact widening."""
    return _quantize("condensa_quantize_bf16", x, want_q, want_dq, stream)


def condensa_dequantize_bf16(q, stream=None):
    return _dequantize("condensa_dequantize_bf16", q, stream)


FP8_E4M3, FP8_E5M2 = 0, 1


def condensa_quantize_fp8(x, fmt, want_q=True, want_dq=True, stream=None):
    """8-bit floating-point codes (uint8; fmt = FP8_E4M3 or FP8_E5M2) and / or their exact widening."""
    import torch
    q = torch.empty(x.shape, dtype=torch.uint8, device=x.device) if want_q else None
    dq = torch.empty_like(x) if want_dq else None
    _check(library().condensa_quantize_fp8(x.data_ptr() if x.numel() else None, x.numel(), int(fmt),
                                           q.data_ptr() if q is not None else None,
                                           dq.data_ptr() if dq is not None else None, _stream(stream)))
    return q, dq


def condensa_dequantize_fp8(q, fmt, stream=None):
    import torch
    dq = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    _check(library().condensa_dequantize_fp8(q.data_ptr() if q.numel() else None, q.numel(), int(fmt), dq.data_ptr(),
                                             _stream(stream)))
    return dq


def condensa_lc_step(tensors, lambdas, mu, density, lambda_out=None, in_place=False, theta=True, grad=True,
                     mask=True, outputs=None, workspace=None, stream=None, pq=False, config=None, nnz=False):
    """Marshals condensa_lc_step.  By default fresh lambda_out tensors are allocated (lambda is left
    untouched); ``in_place`` updates lambda itself.  ``outputs`` may carry preallocated
    theta / grad / mask / lambda_out lists to reuse."""
    import torch
    lib = library()
    dev = tensors[0].device if tensors else torch.device("cuda")
    nt = len(tensors)
    tab = _tensor_table(tensors)
    total = _total(tensors)
    outputs = outputs or {}
    # an output that is switched off is not written, whether or not `outputs` holds buffers for it
    th = (outputs.get("theta") or [torch.empty_like(t) for t in tensors]) if theta else None
    gr = (outputs.get("grad") or [torch.empty_like(t) for t in tensors]) if grad else None
    mk = (outputs.get("mask") or [torch.empty(t.shape, dtype=torch.uint8, device=dev) for t in tensors]) if mask else None
    if in_place:
        lo = None
    else:
        lo = lambda_out or outputs.get("lambda") or [torch.empty_like(t) for t in tensors]
    kl, pl = _ptr_table(lambdas)
    klo, plo = _ptr_table(lo)
    k1, p1 = _ptr_table(th)
    k2, p2 = _ptr_table(gr)
    k3, p3 = _ptr_table(mk)
    results = outputs.get("results")
    if results is None:
        results = torch.zeros((1, len(SELECT_FIELDS)), dtype=torch.int64, device=dev)
    ws, need = _workspace(OP_LC_STEP, total, 0, nt, 1, SCOPE_GLOBAL, dev, workspace, config)
    th16, k4, count = None, None, None
    if pq:
        th16 = outputs.get("theta_f16") or [torch.empty(t.shape, dtype=torch.int16, device=dev) for t in tensors]
        k4, p4 = _ptr_table(th16)
        if nnz:                              # the footprint objective, counted inside the step
            count = outputs.get("nnz")
            if count is None:
                count = torch.zeros(1, dtype=torch.int64, device=dev)
        _check(lib.condensa_lc_step_pq(tab, nt, pl, plo, float(mu), float(density), p1, p4, p2, p3,
                                       None if count is None else count.data_ptr(),
                                       results.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream), _cfg(config)))
    else:
        _check(lib.condensa_lc_step(tab, nt, pl, plo, float(mu), float(density), p1, p2, p3, results.data_ptr(),
                                    ws.data_ptr(), ws.numel(), _stream(stream), _cfg(config)))
    return {"theta": th, "theta_f16": th16, "grad": gr, "mask": mk, "lambda": lambdas if in_place else lo, "nnz": count,
            "results": results, "workspace": ws, "_keep": (kl, klo, k1, k2, k3, k4)}


def condensa_lc_step_pq(tensors, lambdas, mu, density, **kw):
    """condensa_lc_step_pq: the L-C step of the composed prune + fp16 scheme (theta_f16 holds int16 views of the bits)."""
    return condensa_lc_step(tensors, lambdas, mu, density, pq=True, **kw)


def condensa_count_nonzero(tensors, workspace=None, stream=None):
    """Non-zero count of float32 tensors, of 16-bit floating-point codes when the tensors are int16 / float16 /
    bfloat16, or of 8-bit floating-point codes when they are uint8."""
    import torch
    lib = library()
    dev = tensors[0].device if tensors else torch.device("cuda")
    kinds = [(torch.float32,), (torch.int16, torch.float16, torch.bfloat16), (torch.uint8,)]
    kind = next((k for k, ds in enumerate(kinds) if tensors and tensors[0].dtype in ds), 0)
    nt = len(tensors)
    arr = (Tensor * max(nt, 1))()
    for i, t in enumerate(tensors):
        want = kinds[kind]
        if not (t.is_cuda and t.is_contiguous() and t.dtype in want and 1 <= t.dim() <= 4):
            raise TypeError("contiguous device tensors of one element type, 1 to 4 dimensions")
        arr[i].w = t.data_ptr() if t.numel() else None
        for d in range(t.dim()):
            arr[i].shape[d] = t.shape[d]
        arr[i].ndim = t.dim()
    total = _total(tensors)
    count = torch.zeros(1, dtype=torch.int64, device=dev)
    ws, need = _workspace(OP_COUNT_NONZERO, total, 0, nt, 1, SCOPE_GLOBAL, dev, workspace)
    _check(lib.condensa_count_nonzero(arr, nt, kind, count.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream), None))
    return count


def condensa_thin(w, keep_out=None, keep_in=None, keep_out_offset=0, keep_in_offset=0, stream=None):
    """Marshals condensa_thin: ``keep_out`` / ``keep_in`` are device int32 id tensors or None (keep all)."""
    import torch
    lib = library()
    if not (w.is_cuda and w.dtype == torch.float32 and w.is_contiguous() and 2 <= w.dim() <= 4):
        raise TypeError("w must be a contiguous float32 device tensor with 2 to 4 dimensions")
    for k in (keep_out, keep_in):
        if k is not None and not (k.is_cuda and k.dtype == torch.int32 and k.is_contiguous() and k.dim() == 1):
            raise TypeError("keep lists are contiguous 1-D int32 device tensors")
    n_out = w.shape[0] if keep_out is None else keep_out.numel()
    n_in = w.shape[1] if keep_in is None else keep_in.numel()
    out = torch.empty((n_out, n_in) + tuple(w.shape[2:]), dtype=torch.float32, device=w.device)
    if out.numel() == 0:                     # an empty keep list: nothing to gather (NULL would mean "keep all")
        return out
    shape = (ctypes.c_int64 * 4)(*list(w.shape) + [1] * (4 - w.dim()))
    _check(lib.condensa_thin(w.data_ptr() if w.numel() else None, shape, w.dim(),
                             None if keep_out is None else (keep_out.data_ptr() if keep_out.numel() else None),
                             0 if keep_out is None else keep_out.numel(), int(keep_out_offset),
                             None if keep_in is None else (keep_in.data_ptr() if keep_in.numel() else None),
                             0 if keep_in is None else keep_in.numel(), int(keep_in_offset),
                             out.data_ptr() if out.numel() else None, _stream(stream)))
    return out


def condensa_lc_sgd_step(tensors, grad_loss, theta, lambdas, momentum_buf, mu, lr, momentum, workspace=None, stream=None):
    """Marshals condensa_lc_sgd_step: ``tensors`` (weights) and ``momentum_buf`` are updated in place."""
    import torch
    lib = library()
    dev = tensors[0].device if tensors else torch.device("cuda")
    nt = len(tensors)
    tab = _tensor_table(tensors)
    total = _total(tensors)
    k1, p1 = _ptr_table(grad_loss)
    k2, p2 = _ptr_table(theta)
    k3, p3 = _ptr_table(lambdas)
    k4, p4 = _ptr_table(momentum_buf)
    ws, need = _workspace(OP_LC_SGD_STEP, total, 0, nt, 1, SCOPE_GLOBAL, dev, workspace)
    _check(lib.condensa_lc_sgd_step(tab, nt, p1, p2, p3, p4, float(mu), float(lr), float(momentum), ws.data_ptr(),
                                    ws.numel(), _stream(stream), None))
    return ws


STATE_BLOCK = 256                   # elements of a tensor that share the scale of an 8-bit state
TYPE_F32, TYPE_F16, TYPE_BF16 = 0, 1, 2
ROUND_NEAREST, ROUND_STOCHASTIC = 0, 1


def _type_of(dtype):
    import torch
    return {torch.float32: TYPE_F32, torch.float16: TYPE_F16, torch.bfloat16: TYPE_BF16}.get(dtype)


def _device_of(tensors, what):
    """The one device that the tensors of a table lie on; the current one without any."""
    import torch
    devices = {t.device for t in tensors}
    if len(devices) > 1:
        raise TypeError(f"{what} lie on one device")
    return devices.pop() if devices else torch.device("cuda", torch.cuda.current_device())


def _handle_on(device, stream):
    """Handle of the stream of a call for tensors of ``device``: of the given one, which may be any object with a ``cuda_stream``, or of that
    device's current one."""
    if stream is None:
        return _raw_stream()(device.index)
    if getattr(stream, "device", device) != device:
        raise ValueError(f"a stream of {stream.device} for tensors of {device}")
    return int(stream.cuda_stream)


def _stream_on(device, stream):
    """The same as torch's object."""
    import torch
    handle = _handle_on(device, stream)
    if stream is None:
        return torch.cuda.current_stream(device)
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(handle, device=device)


def _wait_unless_captured(stream):
    """A list on the device is read by calls on any stream later on: it is whole before the program goes on."""
    import torch
    with torch.cuda.stream(stream):
        captured = torch.cuda.is_current_stream_capturing()
    if not captured:
        stream.synchronize()


@functools.lru_cache(None)
def _one_device():
    import torch
    return torch.cuda.device_count() == 1


def _run(table, stream, entry, *args):
    """One call of a table's entry point, on the table's device and the given stream (or its handle) or that device's current one."""
    handle = stream if type(stream) is int else _handle_on(table.device, stream)
    if _one_device():
        code = entry(*args, handle)
    else:
        import torch
        if torch.cuda.current_device() == table.index:
            code = entry(*args, handle)
        else:
            with torch.cuda.device(table.index):
                code = entry(*args, handle)
    if code:
        _check(code)


class _Table:
    """What calls on any stream read of a table: the list of descriptors and the tensors that it names."""

    def _holds(self, tensors):
        self._held, self._streams = [t for t in tensors if t is not None], set()

    def keep_for(self, stream):
        """Before a call on a stream, whose handle it returns: what the table holds is not handed out again before the work of that stream is
        done, although table and tensors are dropped.  (A graph that captured a call needs the table for as long as it is replayed.)"""
        handle = _handle_on(self.device, stream)
        if handle not in self._streams:
            stream = _stream_on(self.device, stream)
            for t in self._held:
                t.record_stream(stream)
            self._streams.add(handle)
        return handle


class AdamwTable(_Table):
    """Weights, gradients and states of condensa_lc_adamw_step, laid out on the device once for many steps.  The tensors must
    keep their storage.  See ``adamw_table``."""

    def __init__(self, weights, grads, exp_avg, exp_avg_sq, exp_avg_scale=None, exp_avg_sq_scale=None, theta=None, lambdas=None,
                 codes=None, stream=None):
        import torch
        n = len(weights)
        lists = {"grad": grads, "exp_avg": exp_avg, "exp_avg_sq": exp_avg_sq, "exp_avg_scale": exp_avg_scale,
                 "exp_avg_sq_scale": exp_avg_sq_scale, "theta": theta, "lambda_": lambdas, "codes": codes}
        lists = {k: list(v) for k, v in lists.items() if v is not None}
        if any(len(v) != n for v in lists.values()):
            raise ValueError("every list holds one tensor for each weight")
        bits = 8 if n and exp_avg[0].dtype == torch.uint8 else 32
        state = torch.uint8 if bits == 8 else torch.float32
        if bits == 8 and (exp_avg_scale is None or exp_avg_sq_scale is None):
            raise ValueError("8-bit states come with their scales")
        first = lambda k: next((t for t in lists.get(k, ()) if t is not None), None)  # noqa: E731
        g0, c0 = first("grad"), first("codes")
        grad_type = TYPE_F32 if g0 is None else _type_of(g0.dtype)
        code_type = TYPE_F16 if c0 is None else _type_of(c0.dtype)
        if grad_type is None or code_type in (None, TYPE_F32):
            raise TypeError("gradients are float32, float16 or bfloat16 and codes are float16 or bfloat16")
        want = {"exp_avg": state, "exp_avg_sq": state, "grad": None if g0 is None else g0.dtype, "codes": None if c0 is None else c0.dtype}
        arr = (AdamwTensor * max(n, 1))()
        for i, w in enumerate(weights):
            if not (w.is_cuda and w.dtype == torch.float32 and w.is_contiguous()):
                raise TypeError("weights must be contiguous float32 device tensors")
            arr[i].w = w.data_ptr() or None
            arr[i].n = w.numel()
            for k, v in lists.items():
                t = v[i]
                if t is None and k in ("theta", "lambda_", "codes"):
                    continue
                elems = -(-w.numel() // STATE_BLOCK) if k.endswith("_scale") else w.numel()
                if not (t.device == w.device and t.dtype == want.get(k, torch.float32) and t.is_contiguous() and t.numel() == elems):
                    raise TypeError(f"{k.rstrip('_')} of tensor {i}: a contiguous tensor of {elems} elements beside the weights, one type for all")
                setattr(arr[i], k, t.data_ptr() or None)
        dev = _device_of(weights, "weights")
        lib = library()
        need = int(lib.condensa_adamw_list_bytes(arr, n))
        self._keep = (list(weights), lists)
        self.list = AdamwList()
        st = _stream_on(dev, stream)
        with torch.cuda.stream(st):                                   # its memory too: other streams may not be done with what they freed
            self._memory = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
            _check(lib.condensa_adamw_list_init(arr, n, bits, grad_type, code_type, self._memory.data_ptr(), self._memory.numel(),
                                                int(st.cuda_stream), ctypes.byref(self.list)))
            _wait_unless_captured(st)
        self.ref, self.device, self.index = ctypes.byref(self.list), dev, dev.index
        self._holds([self._memory, *weights, *(t for v in lists.values() for t in v)])


def adamw_table(weights, grads, exp_avg, exp_avg_sq, **kw) -> AdamwTable:
    """The buffers of an AdamW step.  States in 32 bits: float32 ``exp_avg`` and ``exp_avg_sq``.  States in 8 bits: uint8 E4M3 codes,
    with ``exp_avg_scale`` and ``exp_avg_sq_scale`` (float32, one for every 256 elements of a tensor); zeros are a valid start.
    ``theta`` and ``lambdas`` add the L-C penalty, ``codes`` (float16 or bfloat16) receive the updated weights in 16 bits; their
    entries may be None."""
    return AdamwTable(weights, grads, exp_avg, exp_avg_sq, **kw)


def condensa_lc_adamw_step(table: AdamwTable, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, mu=0.0, seed=None,
                           grad_scale=None, stream=None):
    """Marshals condensa_lc_adamw_step: one update of everything in ``table``.  ``seed``: 8-bit states are rounded by random bits
    made from it, another one for every step, best one whose high and low half both change (a counter times an odd 64-bit constant).
    Without one they are rounded to nearest, where a second moment that moves by less than half the distance of two codes in a step,
    which with betas[1] near 1 is all of them, keeps its ratio to the block's largest: give a seed to train with 8-bit states.  States in
    32 bits have nothing that a seed could decide.
    ``grad_scale``: a float32 device scalar."""
    scale = None
    if grad_scale is not None:
        import torch
        if not (grad_scale.get_device() == table.index and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1):
            raise TypeError("grad_scale is one float32 on the device of the weights")
        scale = grad_scale.data_ptr()
    if seed is None or table.list.state_bits == 32:
        rounding, seed = ROUND_NEAREST, 0
    else:
        rounding, seed = ROUND_STOCHASTIC, seed & 0xFFFFFFFFFFFFFFFF
    s = AdamwSettings(lr, betas[0], betas[1], eps, weight_decay, mu, rounding, step, seed, scale, 0)
    _run(table, table.keep_for(stream), library().condensa_lc_adamw_step, table.ref, ctypes.byref(s))


class AdapterTable(_Table):
    """Adapters beside one shared projection, laid out on the device once for many calls.  The tensors must keep their storage.
    See ``adapter_table``."""

    def __init__(self, adapters, grads=None, n_in=None, n_out=None, dtype=None, stream=None):
        import torch
        adapters = [tuple(x) for x in adapters]
        if adapters:
            a0, b0, _ = adapters[0]
            n_in, n_out, dtype = a0.shape[-1], b0.shape[0], a0.dtype
        if grads is not None and len(grads) != len(adapters):
            raise ValueError("gradients: one pair for each adapter")
        if dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("adapters are float16 or bfloat16")
        dev = adapters[0][0].device if adapters else torch.device("cuda", torch.cuda.current_device())
        arr = (Adapter * max(len(adapters), 1))()
        for i, (a, b, scale) in enumerate(adapters):
            r = a.shape[0] if a.dim() == 2 else -1
            for t, shape in ((a, (r, n_in)), (b, (n_out, r))):
                if not (t.is_cuda and t.device == dev and t.dtype == dtype and t.is_contiguous() and tuple(t.shape) == shape):
                    raise TypeError(f"adapter {i}: contiguous A [rank, {n_in}] and B [{n_out}, rank] on one device, one type for all")
            arr[i].a, arr[i].b, arr[i].scale, arr[i].rank = a.data_ptr(), b.data_ptr(), float(scale), r
            if grads is not None:
                ga, gb = grads[i]
                for t, shape in ((ga, (r, n_in)), (gb, (n_out, r))):
                    if not (t.device == dev and t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == shape):
                        raise TypeError(f"gradients of adapter {i}: contiguous float32 tensors shaped like A and B")
                arr[i].grad_a, arr[i].grad_b = ga.data_ptr(), gb.data_ptr()
        lib = library()
        self.dtype, self.device, self.grads = dtype, dev, grads
        self._keep = adapters
        self.list = AdapterList()
        st = _stream_on(dev, stream)
        with torch.cuda.stream(st):                                   # its memory too: other streams may not be done with what they freed
            self._memory = torch.empty(max(int(lib.condensa_adapter_list_bytes(len(adapters))), 256), dtype=torch.uint8, device=dev)
            _check(lib.condensa_adapter_list_init(arr, len(adapters), _type_of(dtype), int(n_in or 0), int(n_out or 0), self._memory.data_ptr(),
                                                  self._memory.numel(), int(st.cuda_stream), ctypes.byref(self.list)))
            _wait_unless_captured(st)
        self.n_in, self.n_out, self.max_rank = self.list.n_in, self.list.n_out, self.list.max_rank
        self.ref, self.index = ctypes.byref(self.list), dev.index
        self._holds([self._memory, *(t for a, b, _ in adapters for t in (a, b)), *(t for pair in grads or () for t in pair)])

    def empty(self, rows, cols):
        import torch
        return torch.empty((rows, cols), dtype=self.dtype, device=self.device)


def adapter_table(adapters, grads=None, **kw) -> AdapterTable:
    """``adapters``: (A [rank, n_in], B [n_out, rank], scale) each, float16 or bfloat16; ``grads``: float32 (grad_A, grad_B) each, which
    condensa_adapter_project_backward writes.  Without any adapter, ``n_in``, ``n_out`` and ``dtype`` describe the projection."""
    return AdapterTable(adapters, grads, **kw)


def adapter_workspace(table: AdapterTable, n_tokens: int, backward: bool = False):
    """Workspace of calls of one direction with ``n_tokens`` tokens or fewer, to be kept between them."""
    import torch
    need = int(library().condensa_adapter_workspace_bytes(ctypes.byref(table.list), int(n_tokens), int(backward)))
    if need == 0:
        raise ValueError("n_tokens is out of range")
    return torch.empty(need, dtype=torch.uint8, device=table.device)


def _made_for(table, stream, make, *args, **kw):
    """A tensor made for a call: on another stream than the current one from that stream's memory, which work that is still under way on the
    current one cannot reach, and not handed out again before the current one, where the program goes on, is done with it."""
    if stream is None:
        return make(*args, **kw)
    import torch
    with torch.cuda.stream(_stream_on(table.device, stream)):
        t = make(*args, **kw)
    t.record_stream(torch.cuda.current_stream(table.device))
    return t


def _rows(name, t, table, n_tokens, width):
    """(address, row stride) of a two-dimensional operand whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if not (len(shape) == 2 and shape[0] == n_tokens and shape[1] == width and t.dtype is table.dtype and t.get_device() == table.index
            and (stride[1] == 1 or width == 1 or n_tokens == 0) and (n_tokens <= 1 or stride[0] >= width)):
        raise TypeError(f"{name}: a {table.dtype} tensor [{n_tokens}, {width}] with contiguous rows, beside the adapters")
    return t.data_ptr(), (stride[0] if n_tokens > 1 else width)      # the address of a tensor without elements is 0


def _token_ids(ids, table, n_tokens):
    if not (ids.dtype is _int32() and ids.get_device() == table.index and ids.is_contiguous() and ids.numel() == n_tokens):
        raise TypeError(f"token_adapter: {n_tokens} contiguous int32 on the device")
    return ids.data_ptr()


@functools.lru_cache(None)
def _int32():
    import torch
    return torch.int32


def _kept_z(z, table, n_tokens):
    shape = z.shape
    if not (len(shape) == 2 and shape[0] == n_tokens and z.dtype is table.dtype and z.get_device() == table.index and z.is_contiguous()):
        raise TypeError(f"z: a contiguous {table.dtype} tensor with a row for each token")
    return z.data_ptr(), shape[1]


def condensa_adapter_project(x, w, table: AdapterTable, token_adapter, y=None, z=False, workspace=None, stream=None):
    """Marshals condensa_adapter_project.  ``z``: a tensor [tokens, >= largest rank] to receive x A^T scale, True to allocate one (the
    backward pass wants it), False for none."""
    T = x.shape[0]
    px, ldx = _rows("x", x, table, T, table.n_in)
    pw, ldw = _rows("w", w, table, table.n_out, table.n_in)
    ids = _token_ids(token_adapter, table, T)
    if y is None:
        y = _made_for(table, stream, table.empty, T, table.n_out)
    py, ldy = _rows("y", y, table, T, table.n_out)
    if z is True:
        z = _made_for(table, stream, table.empty, T, max(table.max_rank, 1))
    z = None if z is False else z
    pz, ldz = (None, 0) if z is None else _kept_z(z, table, T)
    if workspace is None:
        workspace = _made_for(table, stream, adapter_workspace, table, T)
    _run(table, table.keep_for(stream), library().condensa_adapter_project, table.ref, px, ldx, T, pw, ldw, ids, py, ldy, pz, ldz, workspace.data_ptr(),
         workspace.numel())
    return {"y": y, "z": z, "workspace": workspace}


def condensa_adapter_project_backward(dy, x, w, table: AdapterTable, token_adapter, z, dx=True, workspace=None, stream=None):
    """Marshals condensa_adapter_project_backward: writes the gradients that ``table`` names, and ``dx`` (a tensor, True to allocate
    one, False for none)."""
    T = x.shape[0]
    pdy, lddy = _rows("dy", dy, table, T, table.n_out)
    px, ldx = _rows("x", x, table, T, table.n_in)
    pw, ldw = _rows("w", w, table, table.n_out, table.n_in)
    ids = _token_ids(token_adapter, table, T)
    pz, ldz = _kept_z(z, table, T)
    if dx is True:
        dx = _made_for(table, stream, table.empty, T, table.n_in)
    pdx, lddx = (None, 0) if dx is False else _rows("dx", dx, table, T, table.n_in)
    if workspace is None:
        workspace = _made_for(table, stream, adapter_workspace, table, T, backward=True)
    _run(table, table.keep_for(stream), library().condensa_adapter_project_backward, table.ref, pdy, lddy, px, ldx, T, pw, ldw, ids, pz, ldz, pdx, lddx,
         workspace.data_ptr(), workspace.numel())
    return {"dx": None if dx is False else dx, "grads": table.grads, "workspace": workspace}


def condensa_mu_schedule(mu0: float, a: float, j: int) -> float:
    return float(library().condensa_mu_schedule(float(mu0), float(a), int(j)))
