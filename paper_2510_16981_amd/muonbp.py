"""ctypes binding of ``libmuonbp.so`` (C ABI in ``include/muonbp.h``).

Argument marshalling only: every step of the optimizer runs in the HIP
library.  torch supplies device memory (``data_ptr``) and the current HIP
stream.  There is no fallback: if the library is missing, loading raises.
"""

from __future__ import annotations

import ctypes
import os
import struct
from typing import List, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmuonbp.so")

F32, BF16 = 0, 1
E4M3, E5M2 = 0, 1
KERNEL_KINDS = ("momentum", "scale", "pack", "gram", "poly", "apply", "update", "ns_span")
NS_KINDS = ("gram", "poly", "apply")

STATUS = {0: "MUONBP_OK", 1: "MUONBP_E_INVALID", 2: "MUONBP_E_SHAPE",
          3: "MUONBP_E_DTYPE", 4: "MUONBP_E_NOMEM", 5: "MUONBP_E_HIP",
          6: "MUONBP_E_STATE", 7: "MUONBP_E_NONFINITE", 8: "MUONBP_E_TOO_LARGE"}
STATIC_SCRATCH_BYTES = 128 << 20


class MuonBPError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        super().__init__(f"{STATUS.get(status, status)}: {detail}")


class Matrix(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("grid_rows", ctypes.c_int32), ("grid_cols", ctypes.c_int32)]


class Options(ctypes.Structure):
    _fields_ = [("ns_steps", ctypes.c_int32), ("a", ctypes.c_float),
                ("b", ctypes.c_float), ("c", ctypes.c_float),
                ("eps", ctypes.c_float), ("nesterov", ctypes.c_int32),
                ("scale_mode", ctypes.c_int32), ("rms_beta", ctypes.c_float),
                ("param_dtype", ctypes.c_int), ("state_dtype", ctypes.c_int),
                ("ns_dtype", ctypes.c_int), ("tile_policy", ctypes.c_int32),
                ("k_split", ctypes.c_int32), ("coeff_count", ctypes.c_int32),
                ("coeff_table", ctypes.c_float * (3 * 16)), ("stream_hint", ctypes.c_int32),
                ("apply_mode", ctypes.c_int32), ("check_finite", ctypes.c_int32),
                ("device_memory_limit", ctypes.c_int64), ("gram_iteration", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n_problems", ctypes.c_int64), ("n_elements", ctypes.c_int64),
                ("gemm_tiles", ctypes.c_int64 * 3), ("gemm_tile_rows", ctypes.c_int32 * 3),
                ("gemm_tile_cols", ctypes.c_int32 * 3), ("gemm_launches", ctypes.c_int64),
                ("ns_flops", ctypes.c_double),
                ("ns_dense_flops", ctypes.c_double),
                ("elementwise_bytes", ctypes.c_double),
                ("workspace_bytes", ctypes.c_int64),
                ("gemm_split", ctypes.c_int32 * 3), ("apply_nn", ctypes.c_int32),
                ("static_scratch_bytes", ctypes.c_int64), ("device_bytes", ctypes.c_int64),
                ("gram_units", ctypes.c_int64), ("pack_elements", ctypes.c_int64)]


class AdamwOptions(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("max_grad_norm", ctypes.c_float),
                ("param_dtype", ctypes.c_int), ("stream_hint", ctypes.c_int32),
                ("algorithm", ctypes.c_int32)]


class Dense(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("dtype", ctypes.c_int)]


class BlocksRef(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("scale_ld", ctypes.c_int64),
                ("format", ctypes.c_int32)]


class LinearOptions(ctypes.Structure):
    _fields_ = [("workspace_bytes", ctypes.c_int64), ("fp32_sums", ctypes.c_int32)]


class Profile(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 8), ("launches", ctypes.c_int64 * 8),
                ("ms_full_steps", ctypes.c_double * 8),
                ("launches_full_steps", ctypes.c_int64 * 8)]


_lib = None
_torch = None  # set with _lib


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library (raises when it has not been built).

    torch is imported first: its wheel ships its own HIP runtime under the
    same soname as the system one, and the library must bind to the runtime
    that owns torch's memory and streams (loaded the other way round, the
    process would end up with two runtimes)."""
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it with `python -m paper_2510_16981_amd.build`")
    import torch
    _torch = torch
    lib = ctypes.CDLL(path)
    P, I32, I64, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    sig = {
        "muonbp_options_default": (None, [ctypes.POINTER(Options)]),
        "muonbp_create": (ctypes.c_int, [ctypes.POINTER(Matrix), I32, I64, F, F, F, F,
                                         ctypes.POINTER(Options), P, ctypes.POINTER(P)]),
        "muonbp_step": (ctypes.c_int, [P, ctypes.POINTER(P), ctypes.POINTER(P), I64]),
        "muonbp_set_lr": (ctypes.c_int, [P, F, F]),
        "muonbp_set_period": (ctypes.c_int, [P, I64]),
        "muonbp_set_stream": (ctypes.c_int, [P, P]),
        "muonbp_get_momentum": (ctypes.c_int, [P, I32, P]),
        "muonbp_set_momentum": (ctypes.c_int, [P, I32, P]),
        "muonbp_get_update": (ctypes.c_int, [P, I32, P]),
        "muonbp_synchronize": (ctypes.c_int, [P]),
        "muonbp_describe_plan": (ctypes.c_int, [ctypes.POINTER(Matrix), I32,
                                                ctypes.POINTER(Options), I32,
                                                ctypes.POINTER(PlanInfo)]),
        "muonbp_profile_enable": (ctypes.c_int, [P, I32]),
        "muonbp_profile_read": (ctypes.c_int, [P, ctypes.POINTER(Profile)]),
        "muonbp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "muonbp_last_error": (ctypes.c_char_p, [P]),
        "muonbp_destroy": (None, [P]),
        "muonbp_adamw_options_default": (None, [ctypes.POINTER(AdamwOptions)]),
        "muonbp_adamw_create": (ctypes.c_int, [ctypes.POINTER(I64), I32, ctypes.POINTER(AdamwOptions),
                                               P, ctypes.POINTER(P)]),
        "muonbp_adamw_step": (ctypes.c_int, [P, ctypes.POINTER(P), ctypes.POINTER(P), I64, F]),
        "muonbp_adamw_grad_norm": (ctypes.c_int, [P, ctypes.POINTER(F)]),
        "muonbp_adamw_get_state": (ctypes.c_int, [P, I32, P, P]),
        "muonbp_adamw_set_state": (ctypes.c_int, [P, I32, P, P]),
        "muonbp_adamw_set_stream": (ctypes.c_int, [P, P]),
        "muonbp_adamw_synchronize": (ctypes.c_int, [P]),
        "muonbp_adamw_last_error": (ctypes.c_char_p, [P]),
        "muonbp_adamw_destroy": (None, [P]),
        "muonbp_linear_options_default": (None, [ctypes.POINTER(LinearOptions)]),
        "muonbp_linear_create": (ctypes.c_int, [ctypes.POINTER(LinearOptions), P, ctypes.POINTER(P)]),
        "muonbp_linear_quantize": (ctypes.c_int, [P, P, P]),
        "muonbp_linear_quantize_weight": (ctypes.c_int, [P, P, P, P]),
        "muonbp_linear_restore": (ctypes.c_int, [P, P, P]),
        "muonbp_linear_product": (ctypes.c_int, [P, P, P, P, I32]),
        "muonbp_linear_weight_grad": (ctypes.c_int, [P, P, P, P, I32]),
        "muonbp_linear_gated_forward": (ctypes.c_int, [P] * 7),
        "muonbp_linear_gated_backward": (ctypes.c_int, [P] * 8),
        "muonbp_linear_set_stream": (ctypes.c_int, [P, P]),
        "muonbp_linear_synchronize": (ctypes.c_int, [P]),
        "muonbp_linear_last_error": (ctypes.c_char_p, [P]),
        "muonbp_linear_destroy": (None, [P]),
        "muonbp_step_static": (ctypes.c_int, [ctypes.POINTER(Matrix), I32, ctypes.POINTER(P),
                                              ctypes.POINTER(P), P, I64, I64, F, F, F, F,
                                              ctypes.POINTER(Options), P]),
        "muonbp_lr_cosine": (ctypes.c_double, [I64, I64, ctypes.c_double, ctypes.c_double, I64]),
        "muonbp_lr_wsd": (ctypes.c_double, [I64, I64, ctypes.c_double, ctypes.c_double, I64, I64]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


MAX_COEFFS = 16


def options_default(**overrides) -> Options:
    """Library defaults with fields overridden by keyword; ``coeffs`` (a list
    of (a, b, c) triples, one per NS iteration, the last repeated) fills
    coeff_count and coeff_table."""
    o = Options()
    load_library().muonbp_options_default(ctypes.byref(o))
    table = overrides.pop("coeffs", None)
    for k, v in overrides.items():
        if not hasattr(o, k):
            raise AttributeError(k)
        setattr(o, k, v)
    if table is not None:
        if not 1 <= len(table) <= MAX_COEFFS:
            raise ValueError(f"1..{MAX_COEFFS} coefficient triples")
        o.coeff_count = len(table)
        for i, (a, b, c) in enumerate(table):
            o.coeff_table[3 * i:3 * i + 3] = (float(a), float(b), float(c))
    return o


def _mats(mats: Sequence[Tuple[int, int, int, int]]):
    arr = (Matrix * len(mats))()
    for i, (r, c, gr, gc) in enumerate(mats):
        arr[i] = Matrix(r, c, gr, gc)
    return arr


def describe_plan(mats, full: bool, options: Optional[Options] = None) -> PlanInfo:
    """Host-only description of the block (full=False) or full plan."""
    lib = load_library()
    info = PlanInfo()
    st = lib.muonbp_describe_plan(_mats(mats), len(mats),
                                  ctypes.byref(options) if options else None,
                                  int(bool(full)), ctypes.byref(info))
    if st:
        raise MuonBPError(st, "describe_plan")
    return info


def step_static(mats, params: List, grads: List, momentum, step: int, period: int,
                lr_block: float, lr_full: float, mu: float, weight_decay: float = 0.0,
                options: Optional[Options] = None, stream=None) -> None:
    """One allocation-free step (muonbp_step_static): the momentum is the
    caller's ``momentum`` tensor (all matrices back to back, state dtype),
    everything else lives in the library's static scratch array.  Returns
    after the step has completed on ``stream``."""
    import torch
    lib = load_library()
    mats = [tuple(int(v) for v in m) for m in mats]
    n = len(mats)
    if len(params) != n or len(grads) != n:
        raise ValueError("one param and one grad per matrix")
    opts = options if options is not None else options_default()
    total = sum(r * c for r, c, _, _ in mats)
    if not (momentum.is_cuda and momentum.is_contiguous() and momentum.numel() == total
            and momentum.dtype == _torch_dtype(opts.state_dtype)):
        raise ValueError(f"momentum: need a contiguous {_torch_dtype(opts.state_dtype)} CUDA "
                         f"tensor of {total} elements")
    for i, (r, c, _, _) in enumerate(mats):
        for t in (params[i], grads[i]):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(opts.param_dtype)
                    and tuple(t.shape) == (r, c)):
                raise ValueError(f"matrix {i}: need contiguous {_torch_dtype(opts.param_dtype)} "
                                 f"CUDA tensors of shape {(r, c)}")
    if stream is None:
        stream = torch.cuda.current_stream()
    pp = (ctypes.c_void_p * n)(*[p.data_ptr() for p in params])
    gp = (ctypes.c_void_p * n)(*[g.data_ptr() for g in grads])
    st = lib.muonbp_step_static(_mats(mats), n, pp, gp, ctypes.c_void_p(momentum.data_ptr()),
                                int(step), int(period), float(lr_block), float(lr_full), float(mu),
                                float(weight_decay), ctypes.byref(opts),
                                ctypes.c_void_p(stream.cuda_stream))
    if st:
        raise MuonBPError(st, "muonbp_step_static")


def _torch_dtype(code: int):
    import torch
    return {F32: torch.float32, BF16: torch.bfloat16}[code]


class MuonBP:
    """One optimizer context over a fixed list of matrices (Algorithm 1)."""

    def __init__(self, mats: Sequence[Tuple[int, int, int, int]], period: int,
                 lr_block: float, lr_full: float, momentum: float,
                 weight_decay: float = 0.0, options: Optional[Options] = None,
                 stream=None):
        import torch
        self.lib = load_library()
        self.mats = [tuple(int(v) for v in m) for m in mats]
        self.options = options if options is not None else options_default()
        if stream is None:
            stream = torch.cuda.current_stream()
        self._stream = stream
        ctx = ctypes.c_void_p()
        st = self.lib.muonbp_create(_mats(self.mats), len(self.mats), int(period),
                                    float(lr_block), float(lr_full), float(momentum),
                                    float(weight_decay), ctypes.byref(self.options),
                                    ctypes.c_void_p(stream.cuda_stream), ctypes.byref(ctx))
        if st:
            raise MuonBPError(st, "muonbp_create")
        self.ctx = ctx
        self.period = int(period)
        self._ptrs = (ctypes.c_void_p * len(self.mats))()
        self._gptrs = (ctypes.c_void_p * len(self.mats))()

    # -- helpers
    def _check(self, st: int, what: str):
        if st:
            detail = self.lib.muonbp_last_error(self.ctx)
            raise MuonBPError(st, f"{what}: {detail.decode() if detail else ''}")

    def _check_tensor(self, t, i, dtype_code):
        import torch
        r, c = self.mats[i][:2]
        if not (t.is_cuda and t.is_contiguous() and t.dtype == _torch_dtype(dtype_code)
                and tuple(t.shape) == (r, c)):
            raise ValueError(f"matrix {i}: need a contiguous {_torch_dtype(dtype_code)} "
                             f"CUDA tensor of shape {(r, c)}, got {t.dtype} {tuple(t.shape)}")

    def is_full(self, t: int) -> bool:
        return self.period > 0 and t % self.period == 0

    # -- API
    def step(self, params: List, grads: List, t: int) -> None:
        n = len(self.mats)
        if len(params) != n or len(grads) != n:
            raise ValueError("one param and one grad per matrix")
        for i in range(n):
            self._check_tensor(params[i], i, self.options.param_dtype)
            self._check_tensor(grads[i], i, self.options.param_dtype)
            self._ptrs[i] = params[i].data_ptr()
            self._gptrs[i] = grads[i].data_ptr()
        self._check(self.lib.muonbp_step(self.ctx, self._ptrs, self._gptrs, int(t)), "step")

    def set_lr(self, lr_block: float, lr_full: float) -> None:
        self._check(self.lib.muonbp_set_lr(self.ctx, float(lr_block), float(lr_full)), "set_lr")

    def set_period(self, period: int) -> None:
        self._check(self.lib.muonbp_set_period(self.ctx, int(period)), "set_period")
        self.period = int(period)

    def set_stream(self, stream) -> None:
        self._check(self.lib.muonbp_set_stream(self.ctx, ctypes.c_void_p(stream.cuda_stream)),
                    "set_stream")
        self._stream = stream

    def get_momentum(self, i: int, out=None):
        import torch
        r, c = self.mats[i][:2]
        if out is None:
            out = torch.empty((r, c), dtype=_torch_dtype(self.options.state_dtype), device="cuda")
        self._check_tensor(out, i, self.options.state_dtype)
        self._check(self.lib.muonbp_get_momentum(self.ctx, i, ctypes.c_void_p(out.data_ptr())),
                    "get_momentum")
        return out

    def set_momentum(self, i: int, src) -> None:
        self._check_tensor(src, i, self.options.state_dtype)
        self._check(self.lib.muonbp_set_momentum(self.ctx, i, ctypes.c_void_p(src.data_ptr())),
                    "set_momentum")

    def get_update(self, i: int, out=None):
        import torch
        r, c = self.mats[i][:2]
        if out is None:
            out = torch.empty((r, c), dtype=_torch_dtype(self.options.ns_dtype), device="cuda")
        self._check_tensor(out, i, self.options.ns_dtype)
        self._check(self.lib.muonbp_get_update(self.ctx, i, ctypes.c_void_p(out.data_ptr())),
                    "get_update")
        return out

    def synchronize(self) -> None:
        self._check(self.lib.muonbp_synchronize(self.ctx), "synchronize")

    def profile_enable(self, on=True) -> None:
        """True / 1: events around every launch; 2: one span per step over
        the NS GEMM launches (kind "ns_span"); False / 0: off."""
        self._check(self.lib.muonbp_profile_enable(self.ctx, int(on)), "profile_enable")

    def profile_read(self, split: bool = False) -> dict:
        """{kind: (ms, launches)} summed over the launches recorded since the
        last read; with split=True, {"block": {...}, "full": {...}} by the
        kind of step that enqueued them."""
        p = Profile()
        self._check(self.lib.muonbp_profile_read(self.ctx, ctypes.byref(p)), "profile_read")
        if not split:
            return {k: (p.ms[i], p.launches[i]) for i, k in enumerate(KERNEL_KINDS)}
        return {"full": {k: (p.ms_full_steps[i], p.launches_full_steps[i])
                         for i, k in enumerate(KERNEL_KINDS)},
                "block": {k: (p.ms[i] - p.ms_full_steps[i], p.launches[i] - p.launches_full_steps[i])
                          for i, k in enumerate(KERNEL_KINDS)}}

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.muonbp_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- scalar optimizer

def adamw_options_default(**overrides) -> AdamwOptions:
    """Library defaults (beta1 0.9, beta2 0.95, eps 1e-8, weight decay 0.1,
    clipping at 1.0, bf16) with fields overridden by keyword."""
    o = AdamwOptions()
    load_library().muonbp_adamw_options_default(ctypes.byref(o))
    for k, v in overrides.items():
        if not hasattr(o, k):
            raise AttributeError(k)
        setattr(o, k, v)
    return o


class AdamW:
    """AdamW with global-norm clipping over a fixed list of tensors (the
    parameters MuonBP does not orthogonalize)."""

    def __init__(self, sizes: Sequence[int], options: Optional[AdamwOptions] = None, stream=None):
        import torch
        self.lib = load_library()
        self.sizes = [int(n) for n in sizes]
        self.options = options if options is not None else adamw_options_default()
        if stream is None:
            stream = torch.cuda.current_stream()
        arr = (ctypes.c_int64 * len(self.sizes))(*self.sizes)
        ctx = ctypes.c_void_p()
        st = self.lib.muonbp_adamw_create(arr, len(self.sizes), ctypes.byref(self.options),
                                          ctypes.c_void_p(stream.cuda_stream), ctypes.byref(ctx))
        if st:
            raise MuonBPError(st, "muonbp_adamw_create")
        self.ctx = ctx
        self._ptrs = (ctypes.c_void_p * len(self.sizes))()
        self._gptrs = (ctypes.c_void_p * len(self.sizes))()

    def _check(self, st: int, what: str):
        if st:
            detail = self.lib.muonbp_adamw_last_error(self.ctx)
            raise MuonBPError(st, f"{what}: {detail.decode() if detail else ''}")

    def _check_tensor(self, t, i, dtype):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype and t.numel() == self.sizes[i]):
            raise ValueError(f"tensor {i}: need a contiguous {dtype} CUDA tensor of "
                             f"{self.sizes[i]} elements, got {t.dtype} {tuple(t.shape)}")

    def step(self, params: List, grads: List, t: int, lr: float) -> None:
        import torch
        n = len(self.sizes)
        if len(params) != n or len(grads) != n:
            raise ValueError("one param and one grad per tensor")
        dt = _torch_dtype(self.options.param_dtype)
        for i in range(n):
            self._check_tensor(params[i], i, dt)
            self._check_tensor(grads[i], i, dt)
            self._ptrs[i] = params[i].data_ptr()
            self._gptrs[i] = grads[i].data_ptr()
        self._check(self.lib.muonbp_adamw_step(self.ctx, self._ptrs, self._gptrs, int(t), float(lr)),
                    "adamw_step")

    def grad_norm(self) -> float:
        out = ctypes.c_float()
        self._check(self.lib.muonbp_adamw_grad_norm(self.ctx, ctypes.byref(out)), "grad_norm")
        return float(out.value)

    def get_state(self, i: int):
        import torch
        m = torch.empty(self.sizes[i], dtype=torch.float32, device="cuda")
        v = torch.empty_like(m)
        self._check(self.lib.muonbp_adamw_get_state(self.ctx, i, ctypes.c_void_p(m.data_ptr()),
                                                    ctypes.c_void_p(v.data_ptr())), "get_state")
        return m, v

    def set_state(self, i: int, m, v) -> None:
        import torch
        for t in (m, v):
            self._check_tensor(t, i, torch.float32)
        self._check(self.lib.muonbp_adamw_set_state(self.ctx, i, ctypes.c_void_p(m.data_ptr()),
                                                    ctypes.c_void_p(v.data_ptr())), "set_state")

    def synchronize(self) -> None:
        self._check(self.lib.muonbp_adamw_synchronize(self.ctx), "synchronize")

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.muonbp_adamw_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- 8-bit linear layers

BLOCK_COLS, GROUP_COLS = 128, 512


# muonbp_dense and muonbp_blocks as bytes, which take a third of the time of a
# ctypes.Structure to make and are passed by address as they are.
_DENSE = struct.Struct("Pqqqi4x")
_BLOCKS = struct.Struct("PPqqqqi4x")


class Blocks:
    """A matrix in 8-bit floating point with a power-of-two scale for each
    block of 128 columns of a row (muonbp_blocks): ``data`` is uint8, rows x
    (cols rounded up to 128 at least), ``scales`` int32, ceil(cols / 512) x
    rows, a byte for each block.  Holds its tensors; makes no copy."""

    __slots__ = ("_data", "_scales", "_memory", "rows", "cols", "ld", "format", "index", "ref")

    def __init__(self, data, scales, cols: int, format: int = E4M3):
        if _torch is None:
            load_library()
        rows, width = data.shape
        groups, padded = -(-cols // GROUP_COLS), -(-cols // BLOCK_COLS) * BLOCK_COLS
        ld, inner = data.stride()
        index = data.get_device()  # of a CPU tensor: -1
        if data.dtype is not _torch.uint8 or index < 0 or inner != 1 or width < padded:
            raise ValueError(f"data: need a CUDA uint8 matrix with rows of at least {cols} bytes rounded up "
                             f"to {BLOCK_COLS}, got {data.dtype} {tuple(data.shape)}")
        if (scales.shape != (groups, rows) or scales.dtype is not _torch.int32 or scales.get_device() != index
                or (rows > 1 and scales.stride(1) != 1)):
            raise ValueError(f"scales: need an int32 matrix of shape {(groups, rows)} on {data.device}, "
                             f"got {scales.dtype} {tuple(scales.shape)}")
        self._data, self._scales, self._memory = data, scales, None
        self.rows, self.cols, self.format, self.index = rows, cols, format, index
        self.ld = ld = ld if rows > 1 else padded  # of one row: its width may be no multiple of 16
        self.ref = _BLOCKS.pack(data.data_ptr(), scales.data_ptr(), rows, cols, ld,
                                scales.stride(0) if groups > 1 else rows, format)

    @classmethod
    def _in(cls, memory, rows: int, cols: int, ld: int, format: int) -> "Blocks":
        """Blocks in one uint8 tensor: rows x ld bytes, then the scales."""
        self = object.__new__(cls)
        self._data = self._scales = None
        self._memory = memory
        self.rows, self.cols, self.ld, self.format, self.index = rows, cols, ld, format, memory.get_device()
        at = memory.data_ptr()
        self.ref = _BLOCKS.pack(at, at + rows * ld, rows, cols, ld, rows, format)
        return self

    @property
    def data(self):
        if self._data is None:
            self._data = self._memory[:self.rows * self.ld].view(self.rows, self.ld)
        return self._data

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._memory[self.rows * self.ld:].view(_torch.int32).view(
                -(-self.cols // GROUP_COLS), self.rows)
        return self._scales

    def __getitem__(self, rows: slice) -> "Blocks":
        """Rows [a, b) as a matrix of the same memory."""
        a, b, step = rows.indices(self.rows)
        if step != 1:
            raise ValueError("rows of Blocks have step 1")
        return Blocks(self.data[a:max(a, b)], self.scales[:, a:max(a, b)], self.cols, self.format)


class Linear:
    """The 8-bit linear-layer operators on one stream (muonbp_linear_*).

    Matrices are 2-D CUDA tensors with contiguous rows (any row stride of at
    least cols), bf16 or fp32, or ``Blocks``.  Every call is enqueued on the
    context's stream; results not given by ``out`` are allocated on the current
    one.  Where that is another, the call comes after its work so far and before its
    later work, so operands and results are made, used and freed there as with
    torch's own operators (to overlap the two streams, make the context's the
    current one and order them yourself).

    A captured graph that holds calls uses the context's workspace: its replays are
    to be ordered with all other calls and replays of the context, and none may
    follow ``close``.  Results are not part of torch's autograd, whatever the
    operands require.  ``fp32_sums``: products with bf16 results add in fp32 too,
    at half the rate."""

    def __init__(self, workspace_bytes: Optional[int] = None, stream=None, fp32_sums: bool = False):
        import torch
        self.lib = load_library()
        if stream is None:
            stream = torch.cuda.current_stream()
        opts = LinearOptions()
        self.lib.muonbp_linear_options_default(ctypes.byref(opts))
        if workspace_bytes is not None:
            opts.workspace_bytes = int(workspace_bytes)
        opts.fp32_sums = int(fp32_sums)
        ctx = ctypes.c_void_p()
        st = self.lib.muonbp_linear_create(ctypes.byref(opts), ctypes.c_void_p(stream.cuda_stream),
                                           ctypes.byref(ctx))
        if st:
            raise MuonBPError(st, "muonbp_linear_create")
        self.ctx = ctx
        self._stream, self._handle = stream, stream.cuda_stream
        self.device = stream.device
        self._index = stream.device.index
        self._codes = {torch.float32: F32, torch.bfloat16: BF16}
        # The handle of the current stream: torch.cuda.current_stream builds an
        # object for it, which takes longer than the rest of a call.
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)

    # -- helpers
    def _check(self, st: int, what: str):
        if st:
            detail = self.lib.muonbp_linear_last_error(self.ctx)
            raise MuonBPError(st, f"{what}: {detail.decode() if detail else ''}")

    def _join(self):
        """The context's stream waits for the current one, which is another;
        returns the current one, None where the two may not meet."""
        cuda = _torch.cuda
        with cuda.stream(self._stream):
            captured = cuda.is_current_stream_capturing()
        if captured != cuda.is_current_stream_capturing():
            if captured:  # by a program that captures it alone: nothing runs now
                return None
            if self._handle == 0:
                raise ValueError("the default stream cannot be captured: set_stream to the one that is")
        current = cuda.current_stream(self._index)
        self._stream.wait_stream(current)
        return current

    def _run(self, call, what: str, *args):
        if self._current(self._index) == self._handle:
            st = call(self.ctx, *args)
        else:
            current = self._join()
            st = call(self.ctx, *args)
            if current is not None:
                current.wait_stream(self._stream)
        if st:
            self._check(st, what)

    def _dense(self, t, name: str) -> bytes:
        code = self._codes.get(t.dtype)
        if code is None or t.dim() != 2 or t.get_device() != self._index:
            raise ValueError(f"{name}: need a bf16 or fp32 matrix on {self.device}, got {t.dtype} "
                             f"{tuple(t.shape)} on {t.device}")
        rows, cols = t.shape
        ld, inner = t.stride()
        if (inner != 1 and cols > 1) or (ld < cols and rows > 1):
            raise ValueError(f"{name}: need contiguous rows, got strides {t.stride()}")
        return _DENSE.pack(t.data_ptr(), rows, cols, ld if rows > 1 else cols, code)

    def _new(self, rows: int, cols: int, dtype):
        """(A new matrix, its muonbp_dense.)"""
        t = self._empty((rows, cols), dtype)
        code = self._codes.get(dtype)
        if code is None:
            raise ValueError(f"need bf16 or fp32, got {dtype}")
        return t, _DENSE.pack(t.data_ptr(), rows, cols, cols, code)

    def _given(self, out, dtype) -> bytes:
        if dtype is not None and out.dtype != dtype:
            raise ValueError(f"out is {out.dtype}, not {dtype}")
        return self._dense(out, "out")

    def _blocks(self, b: Blocks, name: str) -> bytes:
        if not isinstance(b, Blocks) or b.index != self._index:
            raise ValueError(f"{name}: need Blocks on {self.device}")
        return b.ref

    def _empty(self, shape, dtype):
        return _torch.empty(shape, dtype=dtype, device=self.device)

    def empty_blocks(self, rows: int, cols: int, format: int = E4M3) -> Blocks:
        """Uninitialised Blocks of rows x cols."""
        ld = -(-cols // BLOCK_COLS) * BLOCK_COLS
        return Blocks._in(self._empty(rows * (ld + 4 * -(-cols // GROUP_COLS)), _torch.uint8), rows, cols, ld,
                          format)

    # -- API
    def quantize(self, x, format: Optional[int] = None, out: Optional[Blocks] = None) -> Blocks:
        """x in 8 bits (E4M3, or out's format), one scale for each block of 128
        columns of a row."""
        d = self._dense(x, "x")
        if out is None:
            out = self.empty_blocks(x.shape[0], x.shape[1], E4M3 if format is None else format)
        elif format is not None and out.format != format:
            raise ValueError(f"out is in format {out.format}, not {format}")
        self._run(self.lib.muonbp_linear_quantize, "quantize", d, self._blocks(out, "out"))
        return out

    def quantize_weight(self, w, format: Optional[int] = None, out: Optional[Blocks] = None,
                        out_t: Optional[Blocks] = None) -> Tuple[Blocks, Blocks]:
        """(w, its transpose) in 8 bits (E4M3, or the format of what is given),
        one scale for each 128 x 128 tile."""
        d = self._dense(w, "w")
        rows, cols = w.shape
        given = [b.format for b in (out, out_t) if b is not None]
        if format is None:
            format = given[0] if given else E4M3
        if any(f != format for f in given):
            raise ValueError(f"out and out_t are in formats {given}, not {format}")
        if out is None:
            out = self.empty_blocks(rows, cols, format)
        if out_t is None:
            out_t = self.empty_blocks(cols, rows, format)
        self._run(self.lib.muonbp_linear_quantize_weight, "quantize_weight", d, self._blocks(out, "out"),
                  self._blocks(out_t, "out_t"))
        return out, out_t

    def restore(self, x: Blocks, dtype=None, out=None):
        """The values of x (bf16, or out's type), exact."""
        px = self._blocks(x, "x")
        if out is None:
            out, d = self._new(x.rows, x.cols, dtype or _torch.bfloat16)
        else:
            d = self._given(out, dtype)
        self._run(self.lib.muonbp_linear_restore, "restore", px, d)
        return out

    def _product(self, call, what, pa, pb, rows, cols, dtype, out, accumulate):
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs out")
            out, d = self._new(rows, cols, dtype or _torch.bfloat16)
        else:
            d = self._given(out, dtype)
        self._run(call, what, pa, pb, d, accumulate)
        return out

    def product(self, a: Blocks, b: Blocks, dtype=None, out=None, accumulate: bool = False):
        """a b^T (bf16, or out's type); ``accumulate`` adds it to ``out``."""
        pa, pb = self._blocks(a, "a"), self._blocks(b, "b")
        return self._product(self.lib.muonbp_linear_product, "product", pa, pb, a.rows, b.rows, dtype, out,
                             accumulate)

    def weight_grad(self, x: Blocks, dy, dtype=None, out=None, accumulate: bool = False):
        """x^T dy (bf16, or out's type); ``accumulate`` adds it to ``out``."""
        px, pd = self._blocks(x, "x"), self._dense(dy, "dy")
        return self._product(self.lib.muonbp_linear_weight_grad, "weight_grad", px, pd, x.cols, dy.shape[1], dtype,
                             out, accumulate)

    def gated_forward(self, gate, up, blocks: bool = False, keep: bool = True, format: int = E4M3):
        """(h, gate, up) with h = silu(gate) up of the inputs' dtype (``blocks``:
        in 8 bits) and gate and up kept in 8 bits (None without ``keep``)."""
        g, u = self._dense(gate, "gate"), self._dense(up, "up")
        rows, cols = gate.shape
        d = h8 = g8 = u8 = None
        if blocks:
            h = self.empty_blocks(rows, cols, format)
            h8 = h.ref
        else:
            h, d = self._new(rows, cols, gate.dtype)
        kept = (None, None)
        if keep:
            kept = self.empty_blocks(rows, cols, format), self.empty_blocks(rows, cols, format)
            g8, u8 = kept[0].ref, kept[1].ref
        self._run(self.lib.muonbp_linear_gated_forward, "gated_forward", g, u, d, h8, g8, u8)
        return h, kept[0], kept[1]

    def gated_backward(self, dh, gate: Blocks, up: Blocks, blocks: bool = False, format: int = E4M3):
        """(dgate, dup) of dh's dtype, and with ``blocks`` both in 8 bits too."""
        d = self._dense(dh, "dh")
        pg, pu = self._blocks(gate, "gate"), self._blocks(up, "up")
        rows, cols = dh.shape
        (dgate, a), (dup, b) = self._new(rows, cols, dh.dtype), self._new(rows, cols, dh.dtype)
        if not blocks:
            self._run(self.lib.muonbp_linear_gated_backward, "gated_backward", d, pg, pu, a, b, None, None)
            return dgate, dup
        dgate8, dup8 = self.empty_blocks(rows, cols, format), self.empty_blocks(rows, cols, format)
        self._run(self.lib.muonbp_linear_gated_backward, "gated_backward", d, pg, pu, a, b, dgate8.ref, dup8.ref)
        return dgate, dup, dgate8, dup8

    def set_stream(self, stream) -> None:
        self._check(self.lib.muonbp_linear_set_stream(self.ctx, ctypes.c_void_p(stream.cuda_stream)),
                    "set_stream")
        self._stream, self._handle = stream, stream.cuda_stream

    def synchronize(self) -> None:
        self._check(self.lib.muonbp_linear_synchronize(self.ctx), "synchronize")

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.muonbp_linear_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def lr_cosine(t: int, total: int, lr_max: float, lr_min: float = 0.0, warmup: int = 0) -> float:
    """Cosine schedule of the library (muonbp_lr_cosine)."""
    return load_library().muonbp_lr_cosine(int(t), int(total), float(lr_max), float(lr_min), int(warmup))


def lr_wsd(t: int, total: int, lr_max: float, lr_min: float = 0.0, warmup: int = 0,
           decay: int = 0) -> float:
    """Warmup-stable-decay schedule of the library (muonbp_lr_wsd)."""
    return load_library().muonbp_lr_wsd(int(t), int(total), float(lr_max), float(lr_min), int(warmup),
                                        int(decay))
