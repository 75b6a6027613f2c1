"""ctypes binding of libhack_b200.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/hack.h).  Tensors are passed
as raw device pointers; torch is used by callers for device memory and streams, never here for
arithmetic.  There is no fallback: if the shared library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import operator
import os
import sysconfig
from typing import Optional, Sequence

# HACK_B200_CHECKED=1 selects the checked build of the same sources (bounds checks in the kernels,
# guard rows in the planes); HackCache.close() then also verifies the guard rows.
_CHECKED = os.environ.get("HACK_B200_CHECKED", "0") == "1"
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib",
                         "libhack_b200_checked.so" if _CHECKED else "libhack_b200.so")

HACK_OK, HACK_ERR_INVALID_ARG, HACK_ERR_UNSUPPORTED, HACK_ERR_OOM, HACK_ERR_CUDA, HACK_ERR_STATE, \
    HACK_ERR_TIMEOUT = range(7)
HACK_F32, HACK_BF16 = 0, 1
HACK_OVERFLOW_KEEP_PROTECTED, HACK_OVERFLOW_COMPETE = 0, 1
HACK_OBS_UNIFORM, HACK_OBS_INIT, HACK_OBS_RECENT, HACK_OBS_CALLER, HACK_OBS_FULL = 0, 1, 2, 3, 4
RULE_FRACTION, RULE_RATIO = 0, 1
HACK_ROPE_HALF, HACK_ROPE_PAIRS = 0, 1
HACK_ROPE_PLAIN, HACK_ROPE_LINEAR, HACK_ROPE_BASE, HACK_ROPE_BANDS = 0, 1, 2, 3
HACK_NORM_NONE, HACK_NORM_RMS, HACK_NORM_L2 = 0, 1, 2
HACK_KV4_FEW, HACK_KV4_MANY = 1, 2

EXPORTS = (
    "hack_split_budget", "hack_init_cache", "hack_free_cache", "hack_reset", "hack_set_obs_rows", "hack_get_limits",
    "hack_step_info", "hack_score", "hack_select", "hack_compact", "hack_attend", "hack_attend_variance",
    "hack_classify_heads", "hack_scale_step",
    "hack_scale_step_host", "hack_score_noalloc", "hack_get_lengths", "hack_read_head", "hack_kv_bytes",
    "hack_launch_count", "hack_stage_timing", "hack_stage_times", "hack_poll_status", "hack_set_wait_limit",
    "hack_debug_build", "hack_debug_check", "hack_last_error",
    "hack_rope_plan", "hack_rope", "hack_qk_norm_rope", "hack_scale_step_qkv", "hack_kv4_append", "hack_kv4_read",
    "hack_store_kv4", "hack_kv4_workspace", "hack_kv4_attend", "hack_kv4_poll_status",
)


class HackConfig(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("batch", C.c_int32),
        ("n_scales", C.c_int32), ("scale_sides", C.POINTER(C.c_int32)), ("dtype", C.c_int32),
        ("head_is_contextual", C.POINTER(C.c_uint8)), ("budget_c", C.c_int32), ("budget_s", C.c_int32),
        ("n_obs", C.c_int32), ("n_init_scales", C.c_int32), ("sm_scale", C.c_float),
        ("overflow_policy", C.c_int32), ("device", C.c_int32), ("obs_sampler", C.c_int32),
        ("merge_last", C.c_int32),
    ]


class HackStepInfo(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_new", "stored_c", "stored_s", "cand_c", "cand_s", "kept_c", "kept_s",
        "triggered_c", "triggered_s", "n_obs_rows")]


class HackLimits(C.Structure):
    _fields_ = [("cand_stride", C.c_int32), ("kept_stride", C.c_int32), ("max_new", C.c_int32)]


class HackStrides(C.Structure):
    _fields_ = [("batch", C.c_int64), ("head", C.c_int64), ("token", C.c_int64)]


class HackRopePlan(C.Structure):
    """A rotation: plain data, which hack_rope_plan fills."""
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("axes", C.c_int32),
                ("gain", C.c_float), ("reserved", C.c_int32), ("freq", C.c_double * 64)]


class HackRopeArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("device", "dtype", "batch", "n_heads", "n_tokens", "transpose", "positions_f32",
                                         "reserved")] + [
        ("positions_stride", C.c_int64), ("x", HackStrides), ("y", HackStrides)]


class HackQkvArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("device", "dtype", "batch", "n_heads", "n_kv_heads", "n_tokens", "head_dim",
                                         "norm")] + [
        ("eps", C.c_float), ("positions_f32", C.c_int32), ("positions_stride", C.c_int64)] + [
        (n, HackStrides) for n in ("q", "k", "v", "q_out", "k_out", "v_out")]


class HackKv4Planes(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("device", "batch", "n_kv_heads", "head_dim", "cap", "reserved")] + [("rows", C.c_int64)] + [
        (n, C.c_void_p) for n in ("row_off", "k_codes", "v_codes", "k_scales", "v_scales")]


class HackKv4Rows(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_tokens", C.c_int32), ("k", HackStrides), ("v", HackStrides)]


class HackKv4Attend(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_heads", "n_queries", "max_len", "appended", "causal", "window", "n_sink")] + [
        ("sm_scale", C.c_float), ("wait_polls", C.c_int32), ("workspace_bytes", C.c_int64), ("q", HackStrides), ("out", HackStrides),
        ("form", C.c_int32), ("reserved", C.c_int32)]


class HackError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"hack status {status}: {text}")
        self.status = status


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python paper_2504_09261_b200/build.py` "
            "(there is no fallback implementation)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32 = C.c_void_p, C.c_int32
    lib.hack_last_error.restype = C.c_char_p
    lib.hack_last_error.argtypes = []
    sigs = {
        "hack_split_budget": [i32, C.c_double, i32, C.c_double, i32, C.POINTER(i32), C.POINTER(i32)],
        "hack_init_cache": [C.POINTER(HackConfig), C.POINTER(vp)],
        "hack_free_cache": [vp],
        "hack_reset": [vp],
        "hack_set_obs_rows": [vp, i32, C.POINTER(i32), i32],
        "hack_get_limits": [vp, C.POINTER(HackLimits)],
        "hack_step_info": [vp, i32, i32, C.POINTER(HackStepInfo)],
        "hack_score": [vp, i32, i32, vp, vp, vp, vp],
        "hack_select": [vp, i32, i32, vp, vp, vp, vp],
        "hack_compact": [vp, i32, i32, vp, vp, vp, vp],
        "hack_attend": [vp, i32, i32, vp, vp, vp],
        "hack_attend_variance": [vp, i32, i32, vp, vp, vp, vp],
        "hack_classify_heads": [C.POINTER(C.c_double), i32, i32, C.c_double, C.POINTER(C.c_uint8)],
        "hack_scale_step": [vp, i32, i32, vp, vp, vp, vp, vp],
        "hack_scale_step_host": [vp, i32, i32, vp, vp, vp, vp, vp],
        "hack_score_noalloc": [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, C.c_float, vp],
        "hack_get_lengths": [vp, i32, C.POINTER(i32)],
        "hack_read_head": [vp, i32, i32, i32, i32, vp, C.c_size_t],
        "hack_kv_bytes": [vp, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
        "hack_launch_count": [vp, C.POINTER(C.c_uint64)],
        "hack_poll_status": [vp, vp],
        "hack_set_wait_limit": [vp, C.c_int64],
        "hack_debug_check": [vp, C.POINTER(i32)],
        "hack_stage_timing": [vp, i32],
        "hack_stage_times": [vp, C.POINTER(C.c_double), C.POINTER(C.c_uint64)],
    }
    sigs["hack_rope_plan"] = [i32, i32, i32, i32, C.c_double, i32, C.c_double, C.c_int64, C.c_double, C.c_double, vp]
    sigs["hack_rope"] = [vp] * 6
    sigs["hack_qk_norm_rope"] = [vp] * 14
    sigs["hack_scale_step_qkv"] = [vp, i32, i32] + [vp] * 12
    sigs["hack_kv4_append"] = [vp] * 7
    sigs["hack_kv4_read"] = [vp] * 6
    sigs["hack_store_kv4"] = [vp, i32, vp, vp, vp]
    sigs["hack_kv4_workspace"] = [vp, vp, C.POINTER(C.c_size_t)]
    sigs["hack_kv4_attend"] = [vp] * 8
    sigs["hack_kv4_poll_status"] = [i32, vp]
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.hack_debug_build.argtypes = []
    lib.hack_debug_build.restype = C.c_int32
    return lib


lib = _load()


def _load_call():
    """call(address, handle, layer, scale, *buffers) -> status and run(store, head, address, lead, stream, *tensors) -> status or
    key: the compiled marshalling of the entry points that run step by step (csrc/pycall.c), or the same through ctypes if the module
    was not built for this interpreter."""
    path = os.path.join(os.path.dirname(_LIB_PATH), "_hackcall" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
    if os.path.exists(path):
        spec = importlib.util.spec_from_file_location("_hackcall", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        if hasattr(module, "run"):
            return module.call, module.run
    functions = {_address(n): getattr(lib, n)
                 for n in ("hack_score", "hack_select", "hack_compact", "hack_attend", "hack_attend_variance",
                           "hack_scale_step", "hack_scale_step_host") + _RUN}

    def run(store, head, address, lead, stream, *tensors):
        key = (head,) + tuple(v for x in tensors for v in ((None,) * 4 if x is None else (x.dtype, x.shape, x.stride(), x.get_device())))
        entry = store.get(key)
        return key if entry is None else functions[address](_ptr(lead), entry[1], *map(_ptr, tensors), _ptr(stream))

    return lambda address, handle, layer, scale, *buffers: functions[address](handle, layer, scale, *map(_ptr, buffers)), run


def _address(name: str) -> int:
    return C.cast(getattr(lib, name), C.c_void_p).value


_RUN = ("hack_rope", "hack_qk_norm_rope", "hack_kv4_append", "hack_kv4_read", "hack_kv4_attend")
_call, _run = _load_call()
_SCORE, _SELECT, _COMPACT, _ATTEND, _ATTEND_VARIANCE, _SCALE_STEP, _SCALE_STEP_HOST = map(_address, (
    "hack_score", "hack_select", "hack_compact", "hack_attend", "hack_attend_variance", "hack_scale_step",
    "hack_scale_step_host"))
_ROPE, _QK_NORM_ROPE, _KV4_APPEND, _KV4_READ, _KV4_ATTEND = map(_address, _RUN)


def hack_last_error() -> str:
    return lib.hack_last_error().decode()


def _check(status: int) -> None:
    if status != HACK_OK:
        raise HackError(status, hack_last_error())


def hack_split_budget(budget: int, alpha: float, rule: int, param: float, total_tokens: int):
    bc, bs = C.c_int32(), C.c_int32()
    _check(lib.hack_split_budget(budget, alpha, rule, param, total_tokens, C.byref(bc), C.byref(bs)))
    return bc.value, bs.value


def hack_classify_heads(sigma, n_layers: int, n_heads: int, alpha: float):
    """Head mask (list of n_layers lists of 0/1, 1 = contextual) from the variance matrix."""
    flat = [float(v) for row in sigma for v in (row if hasattr(row, "__iter__") else [row])]
    if len(flat) != n_layers * n_heads:
        raise ValueError("sigma must have n_layers*n_heads entries")
    arr = (C.c_double * len(flat))(*flat)
    out = (C.c_uint8 * len(flat))()
    _check(lib.hack_classify_heads(arr, n_layers, n_heads, alpha, out))
    return [[int(out[l * n_heads + h]) for h in range(n_heads)] for l in range(n_layers)]


def hack_score_noalloc(q, k_cand, scores, n_rows: int, n_queries: int, n_cand: int, score_stride: int,
                       head_dim: int, dtype: int, n_obs: int = 32, sm_scale: float = 0.0, stream=None):
    """Scores on dense device tensors with no device allocation (fixed in-library scratch)."""
    _check(lib.hack_score_noalloc(_ptr(q), _ptr(k_cand), _ptr(scores), n_rows, n_queries, n_cand,
                                  score_stride, head_dim, dtype, n_obs, sm_scale, _ptr(stream)))


def _ptr(x) -> Optional[int]:
    """Raw address of a torch tensor / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


# ------------------------------------------------------------------ tensors [batch, heads, tokens, head_dim]
_DTYPES = {}


def _dtype_of(x) -> int:
    """HACK_F32 or HACK_BF16 of a tensor."""
    d = _DTYPES.get(x.dtype)
    if d is None:
        d = {"torch.float32": HACK_F32, "torch.bfloat16": HACK_BF16}.get(str(x.dtype))
        if d is None:
            raise ValueError(f"dtype {x.dtype}: float32 and bfloat16 are served")
        _DTYPES[x.dtype] = d
    return d


def _strides_of(x, what: str) -> HackStrides:
    s = x.stride()
    if len(s) != 4 or (s[3] != 1 and x.shape[3] != 1):
        raise ValueError(f"{what} must be [batch, heads, tokens, head_dim] with contiguous rows")
    return HackStrides(s[0], s[1], s[2])


def _same(what: str, *tensors) -> None:
    """Same dtype, same device."""
    first = tensors[0]
    for t in tensors[1:]:
        if t is not None and (t.dtype != first.dtype or t.get_device() != first.get_device()):
            raise ValueError(f"{what}: tensors of different types or devices")


def _positions(positions, batch: int, n_tokens: int, axes: int, device: int):
    """(positions_f32, positions_stride) of [tokens(, axes)] or [batch, tokens(, axes)]."""
    f32 = {"torch.int32": 0, "torch.float32": 1}.get(str(positions.dtype))
    if f32 is None:
        raise ValueError("positions must be int32 or float32")
    if positions.get_device() != device or not positions.is_contiguous():
        raise ValueError("positions must be contiguous and on the tensors' device")
    shape, own = tuple(positions.shape), (n_tokens,) if axes == 1 else (n_tokens, axes)
    if shape == own:
        return f32, 0
    if shape == (batch,) + own:
        return f32, n_tokens * axes
    raise ValueError(f"positions of shape {shape}: [batch,] {own} wanted")


def _float_vector(x, n: int, device: int, what: str) -> None:
    if x is not None and (str(x.dtype) != "torch.float32" or x.numel() != n or not x.is_contiguous() or x.get_device() != device):
        raise ValueError(f"{what} must be {n} contiguous float32 values on the tensors' device")


_args_of = {}     # argument structs by shapes, strides and types: they hold nothing of a call's tensors


def _keep(key, args):
    """The struct of a call that is seen for the first time."""
    if len(_args_of) >= 4096:
        _args_of.clear()
    _args_of[key] = (args, C.addressof(args))


def _first(head, args, address, lead, stream, *tensors):
    """A call that found no struct.  head holds plain numbers by now: a tensor of one element, say, would be held by its identity,
    and found again with another value in it."""
    while True:                       # (another thread may empty the store between the two lines below)
        status = _run(_args_of, head, address, lead, stream, *tensors)
        if status.__class__ is not tuple:
            return status
        _keep(status, args)


def hack_rope_plan(head_dim: int, rotary_dim: Optional[int] = None, layout: int = HACK_ROPE_HALF, axes: int = 1,
                   base: float = 10000.0, scaling: int = HACK_ROPE_PLAIN, factor: float = 1.0, trained_length: int = 0,
                   turns_fast: float = 0.0, turns_slow: float = 0.0) -> HackRopePlan:
    plan = HackRopePlan()
    _check(lib.hack_rope_plan(head_dim, head_dim if rotary_dim is None else rotary_dim, layout, axes, base, scaling, factor,
                              trained_length, turns_fast, turns_slow, C.byref(plan)))
    return plan


def hack_rope(plan: HackRopePlan, x, y, positions, transpose: bool = False, stream=None) -> None:
    """y = x rotated to its tokens' positions.  x, y: [batch, heads, tokens, head_dim], any strides but the last; positions:
    int32 or float32 [batch,] tokens[, axes]."""
    head = ("rope", plan.axes, plan.head_dim, transpose)
    status = _run(_args_of, head, _ROPE, C.addressof(plan), stream, x, y, positions)
    if status.__class__ is tuple:
        transpose = bool(transpose)
        status = _first(("rope", plan.axes, plan.head_dim, transpose), _rope_args(plan, x, y, positions, transpose), _ROPE,
                        C.addressof(plan), stream, x, y, positions)
    if status:
        _check(status)


def _rope_args(plan, x, y, positions, transpose):
    _same("hack_rope", x, y)
    b, h, n, d = x.shape
    if tuple(y.shape) != (b, h, n, d) or d != plan.head_dim:
        raise ValueError("x and y must have the same shape, with the plan's head_dim")
    f32, stride = _positions(positions, b, n, plan.axes, x.get_device())
    return HackRopeArgs(x.get_device(), _dtype_of(x), b, h, n, int(transpose), f32, 0, stride, _strides_of(x, "x"),
                        _strides_of(y, "y"))


def _qkv_args(plan, q, k, v, q_out, k_out, v_out, positions, norm, eps, q_weight, k_weight, q_gain, k_gain):
    _same("hack_qk_norm_rope", q, k, v, q_out, k_out, v_out)
    b, h, n, d = q.shape
    kv = k if k is not None else v
    kv_heads = kv.shape[1] if kv is not None else 0
    for t, o, heads, what in ((q, q_out, h, "q"), (k, k_out, kv_heads, "k"), (v, v_out, kv_heads, "v")):
        if (t is None) != (o is None):
            raise ValueError(f"{what} and its output: both or neither")
        if t is not None and (tuple(t.shape) != (b, heads, n, d) or t.shape != o.shape):
            raise ValueError(f"{what}: shapes differ")
    dev = q.get_device()
    _float_vector(q_weight, d, dev, "q_weight")
    _float_vector(k_weight, d, dev, "k_weight")
    _float_vector(q_gain, h, dev, "q_gain")
    _float_vector(k_gain, kv_heads, dev, "k_gain")
    f32, stride = _positions(positions, b, n, plan.axes, dev) if positions is not None and plan is not None else (0, 0)
    none = HackStrides()
    return HackQkvArgs(dev, _dtype_of(q), b, h, kv_heads, n, d, norm, eps, f32, stride,
                       *(none if t is None else _strides_of(t, "a tensor") for t in (q, k, v, q_out, k_out, v_out)))


def hack_qk_norm_rope(plan: Optional[HackRopePlan], q, k, v, q_out, k_out, v_out, positions, norm: int = HACK_NORM_RMS,
                      eps: float = 1e-6, q_weight=None, k_weight=None, q_gain=None, k_gain=None, stream=None) -> None:
    """Queries and keys normalised per head, weighted and rotated, values copied: from views of a projection's output to the
    layout of the steps.  All tensors [batch, heads, tokens, head_dim]; plan and positions None: no rotation."""
    of_plan = None if plan is None else (plan.axes, plan.head_dim)
    lead = None if plan is None else C.addressof(plan)
    status = _run(_args_of, ("qkv", of_plan, norm, eps), _QK_NORM_ROPE, lead, stream, q, k, v, q_out, k_out, v_out, positions, q_weight, k_weight,
                  q_gain, k_gain)
    if status.__class__ is tuple:
        norm, eps = operator.index(norm), float(eps)
        status = _first(("qkv", of_plan, norm, eps),
                        _qkv_args(plan, q, k, v, q_out, k_out, v_out, positions, norm, eps, q_weight, k_weight, q_gain, k_gain),
                        _QK_NORM_ROPE, lead, stream, q, k, v, q_out, k_out, v_out, positions, q_weight, k_weight, q_gain, k_gain)
    if status:
        _check(status)


class HackKv4:
    """A 4-bit cache on the caller's planes: uint8 tensors [rows, head_dim / 2] (codes) and [rows, head_dim / 16] (scales) of K
    and V.  Head i = b * n_kv_heads + h owns cap rows, from row i * cap on, or from row_off[i] (int64, on the device).
    `lens` of the methods: int32 [batch * n_kv_heads] on the device, the rows in use, which is the caller's to keep."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, batch: int, n_kv_heads: int, cap: int, row_off=None):
        dim = 2 * k_codes.shape[-1]
        rows = k_codes.shape[0]
        batch, n_kv_heads, cap = map(operator.index, (batch, n_kv_heads, cap))
        for t, width in ((k_codes, dim // 2), (v_codes, dim // 2), (k_scales, dim // 16), (v_scales, dim // 16)):
            if str(t.dtype) != "torch.uint8" or tuple(t.shape) != (rows, width) or not t.is_contiguous() or \
                    t.get_device() != k_codes.get_device():
                raise ValueError("planes must be contiguous uint8 [rows, head_dim / 2] and [rows, head_dim / 16] on one device")
        if row_off is None:
            if batch * n_kv_heads * cap > rows:
                raise ValueError("the planes have fewer than batch * n_kv_heads * cap rows")
        elif str(row_off.dtype) != "torch.int64" or row_off.numel() != batch * n_kv_heads or not row_off.is_contiguous() or \
                row_off.get_device() != k_codes.get_device():
            raise ValueError("row_off must be batch * n_kv_heads contiguous int64 values on the planes' device")
        self.batch, self.n_kv_heads, self.cap, self.head_dim, self.device = batch, n_kv_heads, cap, dim, k_codes.get_device()
        self._held = (k_codes, k_scales, v_codes, v_scales, row_off)
        self._planes = HackKv4Planes(self.device, batch, n_kv_heads, dim, cap, 0, rows, _ptr(row_off), _ptr(k_codes), _ptr(v_codes),
                                     _ptr(k_scales), _ptr(v_scales))
        self._address = C.addressof(self._planes)
        self._head = (self.device, batch, n_kv_heads, dim)

    def _lengths(self, x, n: int, what: str) -> None:
        if x is not None and (str(x.dtype) != "torch.int32" or x.numel() != n or not x.is_contiguous() or x.get_device() != self.device):
            raise ValueError(f"{what} must be {n} contiguous int32 values on the cache's device")

    def _rows(self, k, v, lens, new_lens):
        self._lengths(lens, self.batch * self.n_kv_heads, "lens")
        self._lengths(new_lens, self.batch, "new_lens")
        _same("4-bit cache", k, v)
        if tuple(k.shape) != tuple(v.shape) or len(k.shape) != 4 or tuple(k.shape[:2]) != (self.batch, self.n_kv_heads) or \
                k.shape[3] != self.head_dim or k.get_device() != self.device:
            raise ValueError("k and v must be [batch, n_kv_heads, tokens, head_dim] on the cache's device")
        return HackKv4Rows(_dtype_of(k), k.shape[2], _strides_of(k, "k"), _strides_of(v, "v"))

    def hack_kv4_append(self, k, v, lens, new_lens=None, stream=None) -> None:
        status = _run(_args_of, self._head, _KV4_APPEND, self._address, stream, k, v, lens, new_lens)
        if status.__class__ is tuple:
            status = _first(self._head, self._rows(k, v, lens, new_lens), _KV4_APPEND, self._address, stream, k, v, lens, new_lens)
        if status:
            _check(status)

    def hack_kv4_read(self, k_out, v_out, first, stream=None) -> None:
        status = _run(_args_of, self._head, _KV4_READ, self._address, stream, k_out, v_out, first)
        if status.__class__ is tuple:
            status = _first(self._head, self._rows(k_out, v_out, first, None), _KV4_READ, self._address, stream, k_out, v_out, first)
        if status:
            _check(status)

    def _attend(self, q, out, lens, max_len, new_lens, appended, causal, n_sink, window, sm_scale, workspace_bytes, form):
        self._lengths(lens, self.batch * self.n_kv_heads, "lens")
        self._lengths(new_lens, self.batch, "new_lens")
        _same("hack_kv4_attend", q, out)
        if tuple(q.shape) != tuple(out.shape) or len(q.shape) != 4 or q.shape[0] != self.batch or q.shape[3] != self.head_dim or \
                q.get_device() != self.device:
            raise ValueError("q and out must be [batch, heads, tokens, head_dim] on the cache's device")
        return HackKv4Attend(_dtype_of(q), q.shape[1], q.shape[2], max_len, int(appended), int(causal), window, n_sink, sm_scale, 0,
                             workspace_bytes, _strides_of(q, "q"), _strides_of(out, "out"), form, 0)

    def hack_kv4_workspace(self, q, max_len: int, causal: bool = False, n_sink: int = 0, window: int = 0, appended: bool = False,
                           form: int = 0) -> int:
        """Bytes of the workspace that hack_kv4_attend needs for queries of this shape and type."""
        need = C.c_size_t()
        args = self._attend(q, q, None, max_len, None, appended, causal, n_sink, window, 0.0, 0, form)
        _check(lib.hack_kv4_workspace(self._address, C.addressof(args), C.byref(need)))
        return need.value

    def hack_kv4_attend(self, q, out, lens, max_len: int, workspace=None, new_lens=None, appended: bool = False, causal: bool = False,
                        n_sink: int = 0, window: int = 0, sm_scale: float = 0.0, form: int = 0, stream=None) -> None:
        """q, out: [batch, heads, tokens, head_dim].  max_len: any bound of the lengths (one that is rounded up, rather than another
        in every step, spares the host a new argument struct).  workspace: a uint8 tensor of hack_kv4_workspace bytes, or None
        where that is 0."""
        head = (self._head, max_len, appended, causal, n_sink, window, sm_scale, form)
        status = _run(_args_of, head, _KV4_ATTEND, self._address, stream, q, out, lens, new_lens, workspace)
        if status.__class__ is tuple:
            room = 0 if workspace is None else workspace.numel() * workspace.element_size()
            if room and (not workspace.is_contiguous() or workspace.get_device() != self.device):
                raise ValueError("the workspace must be contiguous and on the cache's device")
            max_len, n_sink, window, form = map(operator.index, (max_len, n_sink, window, form))
            appended, causal, sm_scale = bool(appended), bool(causal), float(sm_scale)
            status = _first((self._head, max_len, appended, causal, n_sink, window, sm_scale, form),
                            self._attend(q, out, lens, max_len, new_lens, appended, causal, n_sink, window, sm_scale, room, form),
                            _KV4_ATTEND, self._address, stream, q, out, lens, new_lens, workspace)
        if status:
            _check(status)

    def hack_kv4_poll_status(self, stream=None) -> None:
        _check(lib.hack_kv4_poll_status(self.device, _ptr(stream)))


class HackCache:
    """Owner of one hack_cache_t.  Methods mirror the C entry points of the same name."""

    def __init__(self, n_layers: int, n_heads: int, head_dim: int, batch: int, sides: Sequence[int],
                 dtype: int, head_is_contextual, budget_c: int, budget_s: int, n_obs: int = 32,
                 n_init_scales: int = 2, sm_scale: float = 0.0,
                 overflow_policy: int = HACK_OVERFLOW_KEEP_PROTECTED, device: int = 0,
                 obs_sampler: int = HACK_OBS_UNIFORM, merge_last: bool = False):
        self._h = C.c_void_p()
        sides_arr = (C.c_int32 * len(sides))(*[int(s) for s in sides])
        flat = [int(v) for v in (head_is_contextual.reshape(-1).tolist()
                                 if hasattr(head_is_contextual, "reshape") else head_is_contextual)]
        mask_arr = (C.c_uint8 * len(flat))(*flat)
        if len(flat) != n_layers * n_heads:
            raise ValueError("head_is_contextual must have n_layers*n_heads entries")
        cfg = HackConfig(n_layers, n_heads, head_dim, batch, len(sides), sides_arr, dtype, mask_arr,
                         budget_c, budget_s, n_obs, n_init_scales, sm_scale, overflow_policy, device,
                         obs_sampler, 1 if merge_last else 0)
        _check(lib.hack_init_cache(C.byref(cfg), C.byref(self._h)))
        self._address = self._h.value
        self.n_layers, self.n_heads, self.head_dim, self.batch = n_layers, n_heads, head_dim, batch
        self.dtype = dtype
        self.elt = 4 if dtype == HACK_F32 else 2
        lim = HackLimits()
        _check(lib.hack_get_limits(self._h, C.byref(lim)))
        self.cand_stride, self.kept_stride, self.max_new = lim.cand_stride, lim.kept_stride, lim.max_new

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            problem = None
            if lib.hack_debug_build():
                # checked build: no kernel may have tripped a bounds check or touched a guard row
                if lib.hack_poll_status(self._h, None) != HACK_OK:
                    problem = hack_last_error()
                bad = C.c_int32()
                if lib.hack_debug_check(self._h, C.byref(bad)) == HACK_OK and bad.value and problem is None:
                    problem = f"{bad.value} guard rows overwritten: {hack_last_error()}"
            lib.hack_free_cache(self._h)
            self._h = C.c_void_p()
            self._address = 0
            if problem:
                raise HackError(HACK_ERR_STATE, problem)

    def hack_debug_check(self) -> int:
        bad = C.c_int32()
        _check(lib.hack_debug_check(self._h, C.byref(bad)))
        return bad.value

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def hack_set_obs_rows(self, scale: int, rows: Sequence[int]) -> None:
        arr = (C.c_int32 * len(rows))(*[int(r) for r in rows])
        _check(lib.hack_set_obs_rows(self._h, scale, arr, len(rows)))

    def hack_reset(self) -> None:
        _check(lib.hack_reset(self._h))

    def hack_step_info(self, layer: int, scale: int) -> HackStepInfo:
        info = HackStepInfo()
        _check(lib.hack_step_info(self._h, layer, scale, C.byref(info)))
        return info

    def hack_score(self, layer, scale, q, k_new, scores, stream=None) -> None:
        _check(_call(_SCORE, self._address, layer, scale, q, k_new, scores, stream))

    def hack_select(self, layer, scale, scores, idx, kept_out=None, stream=None) -> None:
        _check(_call(_SELECT, self._address, layer, scale, scores, idx, kept_out, stream))

    def hack_compact(self, layer, scale, idx, k_new, v_new, stream=None) -> None:
        _check(_call(_COMPACT, self._address, layer, scale, idx, k_new, v_new, stream))

    def hack_attend(self, layer, scale, q, out, stream=None) -> None:
        _check(_call(_ATTEND, self._address, layer, scale, q, out, stream))

    def hack_attend_variance(self, layer, scale, q, out, sigma, stream=None) -> None:
        _check(_call(_ATTEND_VARIANCE, self._address, layer, scale, q, out, sigma, stream))

    def hack_scale_step(self, layer, scale, q, k, v, out, stream=None) -> None:
        status = _call(_SCALE_STEP, self._address, layer, scale, q, k, v, out, stream)
        if status:
            _check(status)

    def hack_scale_step_host(self, layer, scale, q, k, v, out, stream=None) -> None:
        _check(_call(_SCALE_STEP_HOST, self._address, layer, scale, q, k, v, out, stream))

    def hack_scale_step_qkv(self, layer, scale, plan: Optional[HackRopePlan], q, k, v, out, positions, norm: int = HACK_NORM_RMS,
                            eps: float = 1e-6, q_weight=None, k_weight=None, q_gain=None, k_gain=None, stream=None) -> None:
        """hack_qk_norm_rope into buffers of the cache, then hack_scale_step."""
        args = _qkv_args(plan, q, k, v, q, k, v, positions, norm, eps, q_weight, k_weight, q_gain, k_gain)
        _check(lib.hack_scale_step_qkv(self._h, layer, scale, None if plan is None else C.addressof(plan), C.addressof(args), _ptr(q), _ptr(k),
                                       _ptr(v), _ptr(positions), _ptr(q_weight), _ptr(k_weight), _ptr(q_gain), _ptr(k_gain), _ptr(out),
                                       _ptr(stream)))

    def hack_store_kv4(self, layer: int, kv4: HackKv4, lens, stream=None) -> None:
        kv4._lengths(lens, self.batch * self.n_heads, "lens")
        _check(lib.hack_store_kv4(self._h, layer, kv4._address, _ptr(lens), _ptr(stream)))

    def hack_get_lengths(self, layer: int):
        n = self.batch * self.n_heads
        arr = (C.c_int32 * n)()
        _check(lib.hack_get_lengths(self._h, layer, arr))
        return list(arr)

    def hack_read_head(self, layer: int, b: int, h: int, which: int) -> bytes:
        length = self.hack_get_lengths(layer)[b * self.n_heads + h]
        nbytes = length * (4 if which == 2 else self.head_dim * self.elt)
        buf = C.create_string_buffer(max(nbytes, 1))
        _check(lib.hack_read_head(self._h, layer, b, h, which, buf, nbytes))
        return buf.raw[:nbytes]

    def hack_kv_bytes(self):
        live, peak, res = C.c_size_t(), C.c_size_t(), C.c_size_t()
        _check(lib.hack_kv_bytes(self._h, C.byref(live), C.byref(peak), C.byref(res)))
        return live.value, peak.value, res.value

    def hack_launch_count(self) -> int:
        n = C.c_uint64()
        _check(lib.hack_launch_count(self._h, C.byref(n)))
        return n.value

    def hack_stage_timing(self, enable: bool) -> None:
        _check(lib.hack_stage_timing(self._h, 1 if enable else 0))

    def hack_stage_times(self):
        ms = (C.c_double * 4)()
        n = (C.c_uint64 * 4)()
        _check(lib.hack_stage_times(self._h, ms, n))
        names = ("score", "select", "compact", "attend")
        return {k: (ms[i], n[i]) for i, k in enumerate(names)}

    def hack_set_wait_limit(self, cycles: int) -> None:
        _check(lib.hack_set_wait_limit(self._h, cycles))

    def hack_poll_status(self, stream=None) -> None:
        _check(lib.hack_poll_status(self._h, _ptr(stream)))
