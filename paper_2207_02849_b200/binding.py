"""ctypes binding of include/betty.h.  Argument marshalling only: every computation runs in
the CUDA library.  torch is used for device memory and the current stream."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))

# ---- enums (mirrors of betty.h) ----
BETTY_OK = 0
(BETTY_ERR_INVALID_ARG, BETTY_ERR_SHAPE, BETTY_ERR_DTYPE, BETTY_ERR_ALIGNMENT, BETTY_ERR_WORKSPACE,
 BETTY_ERR_CUDA, BETTY_ERR_NONFINITE, BETTY_ERR_BREAKDOWN, BETTY_ERR_TIMEOUT,
 BETTY_ERR_UNSUPPORTED, BETTY_ERR_CAPACITY) = range(1, 12)
(LOSS_LOGREG_WD, LOSS_LOGREG, LOSS_QUADRATIC_WD, LOSS_QUADRATIC, LOSS_MLP_CE_REWEIGHT, LOSS_MLP_CE,
 LOSS_WEIGHTNET_DETECT, LOSS_MLP_CE_CORRECT) = range(8)
PARAM_VECTOR, PARAM_MLP, PARAM_WEIGHTNET, PARAM_LOGWD, PARAM_CORRECTNET = range(5)
BETTY_NEUMANN, BETTY_CG, BETTY_FD = range(3)
ACT_RELU, ACT_GELU, ACT_SILU = range(3)
NORM_NONE, NORM_RMS, NORM_LAYER = range(3)
GATE_NONE, GATE_LINEAR, GATE_SIGMOID = range(3)
BETTY_F32, BETTY_BF16, BETTY_I32, BETTY_F16, BETTY_I64 = range(5)
BETTY_OPT_GD, BETTY_OPT_MOMENTUM, BETTY_OPT_ADAM = range(3)
BETTY_LR_CONSTANT, BETTY_LR_MULTISTEP, BETTY_LR_COSINE = range(3)


class BettyError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {betty_status_string(status)} (status {status})")


class _MethodCfg(C.Structure):
    _fields_ = [("method", C.c_int32), ("K", C.c_int32), ("alpha", C.c_float), ("eps0", C.c_float),
                ("tol", C.c_float)]


_ALLREDUCE = C.CFUNCTYPE(C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p)


class _Comm(C.Structure):
    _fields_ = [("allreduce", _ALLREDUCE), ("user", C.c_void_p), ("row_weight", C.c_float)]


class _Level(C.Structure):
    pass


_Level._fields_ = [
    ("loss", C.c_int32), ("param_kind", C.c_int32), ("params", C.c_void_p), ("n_params", C.c_int64),
    ("X", C.c_void_p), ("x_dtype", C.c_int32), ("n", C.c_int64), ("d", C.c_int64),
    ("y", C.c_void_p), ("aux", C.c_void_p), ("n_layers", C.c_int32), ("widths", C.POINTER(C.c_int64)),
    ("activation", C.c_int32), ("lr", C.c_float), ("mu", C.c_float), ("optimizer", C.c_int32),
    ("momentum", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("adam_eps", C.c_float),
    ("weight_decay", C.c_float), ("opt_state", C.c_void_p), ("n_constraints", C.c_int32),
    ("constraints", C.POINTER(C.POINTER(_Level))),
    ("lr_schedule", C.c_int32), ("lr_step0", C.c_int32), ("lr_t_max", C.c_int32), ("lr_milestones", C.c_int32 * 4),
    ("lr_gamma", C.c_float), ("lr_min", C.c_float), ("grad_accum", C.c_int32), ("comm", C.POINTER(_Comm)),
    ("precision", C.c_int32), ("loss_scale", C.c_void_p),
]

class _Edge(C.Structure):
    _fields_ = [("src", C.c_int32), ("dst", C.c_int32)]


class _GemmOperands(C.Structure):
    _fields_ = [("A", C.c_void_p), ("lda", C.c_int64), ("a_transposed", C.c_int32), ("B", C.c_void_p),
                ("ldb", C.c_int64), ("b_transposed", C.c_int32), ("K", C.c_int32), ("alpha", C.c_float)]


class _BlockNormCfg(C.Structure):
    _fields_ = [("d", C.c_int64), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("pre", C.c_int32), ("post", C.c_int32),
                ("gate", C.c_int32), ("bias", C.c_int32), ("rows_per_gate", C.c_int64), ("eps", C.c_float)]


class _GroupedCfg(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("dtype", C.c_int32), ("n_in", C.c_int64), ("n_out", C.c_int64)]


class _Act8Cfg(C.Structure):
    _fields_ = [("cols", C.c_int64), ("dtype", C.c_int32), ("act", C.c_int32), ("gated", C.c_int32)]


class _VocabCfg(C.Structure):
    _fields_ = [("vocab", C.c_int64), ("d", C.c_int64), ("dtype", C.c_int32), ("temperature", C.c_float), ("smoothing", C.c_float),
                ("z_loss", C.c_float)]


_lib = None


def lib_path() -> str:
    return os.path.join(_HERE, "libbetty.so")


def lib():
    """The loaded CUDA library.  Raises if it has not been built: nothing here falls back to
    another implementation."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2207_02849_b200.build` "
                           "(nvcc, sm_100a); this package has no CPU fallback")
    L = C.CDLL(path)
    LP, VP, I32, SZ, F = C.POINTER(_Level), C.c_void_p, C.c_int32, C.c_size_t, C.c_float
    sig = {
        "betty_workspace_size": [C.POINTER(LP), I32, C.POINTER(SZ)],
        "betty_reset_status": [VP, SZ, VP],
        "betty_poll_status": [VP, VP, C.POINTER(I32)],
        "betty_lower_step": [LP, I32, VP, SZ, VP],
        "betty_grad": [LP, LP, VP, VP, SZ, VP],
        "betty_hvp": [LP, VP, VP, VP, SZ, VP],
        "betty_mixed_vjp": [LP, LP, VP, VP, VP, SZ, VP],
        "betty_hypergrad_neumann": [LP, LP, LP, I32, F, VP, VP, SZ, VP],
        "betty_hypergrad_cg": [LP, LP, LP, I32, F, VP, VP, SZ, VP],
        "betty_hypergrad_fd": [LP, LP, LP, F, F, VP, VP, SZ, VP],
        "betty_hypergrad_itd": [LP, LP, LP, I32, VP, VP, SZ, VP],
        "betty_chain_levels": [C.POINTER(LP), I32, C.POINTER(I32), I32, C.POINTER(_MethodCfg), VP, VP, I32,
                               VP, SZ, VP],
    }
    sig["betty_hvp_logreg_static"] = [VP, C.c_int64, C.c_int64, VP, VP, VP, VP, VP, VP]
    sig["betty_gemm_bf16"] = [I32, I32, I32, C.POINTER(_GemmOperands), VP, C.c_int64, F, I32, VP, SZ, VP]
    I64, BN, A8 = C.c_int64, C.POINTER(_BlockNormCfg), C.POINTER(_Act8Cfg)
    mat = [VP, I64]
    sig["betty_block_norm"] = [BN, VP, I64] + 5 * mat + [VP]
    sig["betty_block_norm_workspace_size"] = [BN, I64, C.POINTER(SZ)]
    sig["betty_block_norm_workspace_size_for"] = [BN, I64, I32, C.POINTER(SZ)]
    sig["betty_block_norm_backward"] = [BN, VP, I64] + 8 * mat + [VP, VP, SZ, VP]
    sig["betty_act8_store"] = [A8, I64] + 4 * mat + [VP]
    sig["betty_act8_restore"] = [A8, I64] + 3 * mat + [VP]
    sig["betty_act8_backward"] = [A8, I64] + 5 * mat + [VP]
    GC = C.POINTER(_GroupedCfg)
    sig["betty_grouped_workspace_size"] = [GC, I64, I32, C.POINTER(SZ)]
    sig["betty_grouped_forward"] = sig["betty_grouped_backward_data"] = [GC, I64, VP] + 2 * mat + [I64] + mat + [I32, VP, SZ, VP]
    sig["betty_grouped_backward_weight"] = [GC, I64, VP] + 3 * mat + [I64, I32, VP, SZ, VP]
    VC = C.POINTER(_VocabCfg)
    sig["betty_vocab_workspace_size"] = [VC, I64, I32, I32, C.POINTER(SZ)]
    head, top, results = [VC, I64] + 2 * mat, [I32] + mat + [I32] + mat + [I32], mat + [I32] + mat + [I32]
    sig["betty_vocab_ce"] = head + [VP, I32, VP, VP, VP, SZ, VP]
    sig["betty_vocab_ce_backward"] = head + [VP, I32, VP, VP] + results + [VP, SZ, VP]
    sig["betty_vocab_distill"] = head + top + [VP, VP, VP, SZ, VP]
    sig["betty_vocab_distill_backward"] = head + top + [VP, VP] + results + [VP, SZ, VP]
    EP, IP = C.POINTER(_Edge), C.POINTER(I32)
    sig["betty_find_paths"] = [I32, EP, I32, EP, I32, I32, IP, I32, IP, I32, IP, IP]
    sig["betty_selftest_wait_timeout"] = [VP, SZ, VP]
    sig["betty_engine_run"] = [C.POINTER(LP), I32, EP, I32, EP, I32, C.POINTER(_MethodCfg), IP, I32, IP, I32, IP, VP, SZ, VP]
    sig["betty_hypergrad_graph"] = [C.POINTER(LP), I32, EP, I32, EP, I32, I32, C.POINTER(_MethodCfg), VP, VP, SZ, VP]
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, C.c_int
    L.betty_status_string.argtypes, L.betty_status_string.restype = [C.c_int], C.c_char_p
    L.betty_kernel_launches.argtypes, L.betty_kernel_launches.restype = [], C.c_uint64
    L.betty_selftest_smem_limit.argtypes = [I32, I32, C.c_uint64]
    L.betty_selftest_smem_limit.restype = I32
    _lib = L
    return L


def betty_status_string(status: int) -> str:
    return lib().betty_status_string(int(status)).decode()


def betty_kernel_launches() -> int:
    return int(lib().betty_kernel_launches())


_comm_error = [None]      # exception raised inside a data-parallel all-reduce callback, if any


def _check(status: int, where: str):
    if status != BETTY_OK:
        cause, _comm_error[0] = _comm_error[0], None
        if cause is not None:
            raise BettyError(status, where) from cause
        raise BettyError(status, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device tensors must be contiguous CUDA tensors")
    return t.data_ptr()


_raw_stream, _raw_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())       # the handle without the Stream object around it: 0.2 us instead of 3.2
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_DT = {torch.float32: BETTY_F32, torch.bfloat16: BETTY_BF16, torch.int32: BETTY_I32, torch.float16: BETTY_F16}


class Level:
    """Host-side descriptor of one problem P_k: keeps the tensors alive and owns the C struct."""

    def __init__(self, loss: int, param_kind: int, params: torch.Tensor, X: Optional[torch.Tensor] = None,
                 y: Optional[torch.Tensor] = None, aux: Optional[torch.Tensor] = None,
                 widths: Optional[Sequence[int]] = None, activation: int = ACT_RELU, lr: float = 0.1,
                 mu: float = 0.0):
        self.params, self.X, self.y, self.aux = params, X, y, aux
        self.widths = tuple(int(w) for w in widths) if widths is not None else None
        self.constraints: list[Level] = []
        s = _Level()
        s.loss, s.param_kind = int(loss), int(param_kind)
        s.params, s.n_params = _ptr(params), params.numel()
        s.X = _ptr(X)
        s.x_dtype = _DT.get(X.dtype, -1) if X is not None else BETTY_F32
        s.n, s.d = (X.shape[0], X.shape[1]) if X is not None else (0, 0)
        s.y, s.aux = _ptr(y), _ptr(aux)
        if self.widths is not None:
            self._widths = (C.c_int64 * len(self.widths))(*self.widths)
            s.n_layers, s.widths = len(self.widths) - 1, self._widths
        else:
            s.n_layers, s.widths = 0, None
        s.activation, s.lr, s.mu = int(activation), float(lr), float(mu)
        s.optimizer, s.opt_state = BETTY_OPT_GD, None
        self.opt_state = None
        s.n_constraints, s.constraints = 0, None
        self.c = s

    def set_constraints(self, levels: Sequence["Level"]) -> "Level":
        self.constraints = list(levels)
        self._carr = (C.POINTER(_Level) * max(1, len(levels)))(*[C.pointer(l.c) for l in levels])
        self.c.n_constraints = len(levels)
        self.c.constraints = self._carr if levels else None
        return self

    def set_optimizer(self, kind: int, momentum: float = 0.0, beta1: float = 0.9, beta2: float = 0.999,
                      eps: float = 1e-8, weight_decay: float = 0.0) -> "Level":
        """Chooses the optimiser of this problem's steps and allocates its zero-initialised state."""
        n = self.params.numel()
        size = {BETTY_OPT_GD: 0, BETTY_OPT_MOMENTUM: n, BETTY_OPT_ADAM: 2 * n + 1}[int(kind)]
        self.opt_state = torch.zeros(max(size, 1), dtype=torch.float32, device=self.params.device) if size else None
        self.c.optimizer, self.c.momentum = int(kind), float(momentum)
        self.c.beta1, self.c.beta2, self.c.adam_eps = float(beta1), float(beta2), float(eps)
        self.c.weight_decay = float(weight_decay)
        self.c.opt_state = _ptr(self.opt_state)
        return self

    def set_lr_schedule(self, kind: int, step0: int = 0, milestones: Sequence[int] = (), gamma: float = 0.1,
                        t_max: int = 1, lr_min: float = 0.0) -> "Level":
        """Step size as a function of the steps taken (betty_lr_schedule); step0 = steps taken before the
        next call."""
        if len(milestones) > 4:
            raise ValueError("at most 4 milestones")
        self.c.lr_schedule, self.c.lr_step0, self.c.lr_t_max = int(kind), int(step0), int(t_max)
        for i in range(4):
            self.c.lr_milestones[i] = int(milestones[i]) if i < len(milestones) else 0
        self.c.lr_gamma, self.c.lr_min = float(gamma), float(lr_min)
        return self

    def set_comm(self, allreduce, row_weight: float) -> "Level":
        """Marks this level as one rank's share of its problem's batch (betty_comm).  `allreduce(ptr, count,
        stream)` must sum `count` floats at device address `ptr` over all ranks, in place, ordered on the
        CUDA stream handle `stream`; an exception it raises surfaces as BETTY_ERR_CUDA from the library call
        (and is re-raised by the binding).  row_weight = this rank's rows / all rows.  None removes it."""
        if allreduce is None:
            self._comm = self._comm_cb = None
            self.c.comm = None
            return self
        self.comm_error = None

        def _cb(user, buf, count, stream):
            try:
                allreduce(int(buf), int(count), int(stream or 0))
                return 0
            except BaseException as e:           # never let an exception cross the C frames
                self.comm_error = _comm_error[0] = e
                return 1
        self._comm_cb = _ALLREDUCE(_cb)
        self._comm = _Comm(self._comm_cb, None, float(row_weight))
        self.c.comm = C.pointer(self._comm)
        return self

    def set_precision(self, dtype: int) -> "Level":
        """Operand type of an MLP block's matrix products: BETTY_BF16 (default) or BETTY_F16."""
        self.c.precision = int(dtype)
        return self

    def set_loss_scale(self, scale: Optional[float], growth_interval: int = 0) -> "Level":
        """Loss scaling of the lower steps of a BETTY_F16 block: allocates the four-float device state
        [scale, good steps, growth interval, skipped steps] (see betty.h); None switches it off."""
        if scale is None:
            self.loss_scale_state = None
            self.c.loss_scale = None
            return self
        self.loss_scale_state = torch.tensor([float(scale), 0.0, float(growth_interval), 0.0], dtype=torch.float32,
                                             device=self.params.device)
        self.c.loss_scale = _ptr(self.loss_scale_state)
        return self

    def set_grad_accum(self, n_micro: int) -> "Level":
        """Steps of this problem average the gradients of n_micro equal micro-batches of its batch."""
        self.c.grad_accum = int(n_micro)
        return self

    @property
    def ref(self):
        return C.byref(self.c)


class MethodCfg:
    def __init__(self, method: int, K: int = 0, alpha: float = 1.0, eps0: float = 0.01, tol: float = 0.0):
        self.c = _MethodCfg(int(method), int(K), float(alpha), float(eps0), float(tol))


def _level_array(levels: Sequence[Level]):
    return (C.POINTER(_Level) * len(levels))(*[C.pointer(l.c) for l in levels])


def betty_workspace_size(levels: Sequence[Level]) -> int:
    out = C.c_size_t(0)
    _check(lib().betty_workspace_size(_level_array(levels), len(levels), C.byref(out)), "betty_workspace_size")
    return int(out.value)


class Workspace:
    """Caller-owned scratch (a torch uint8 tensor) sized by betty_workspace_size."""

    def __init__(self, levels: Sequence[Level], device="cuda", extra_bytes: int = 0):
        self.nbytes = betty_workspace_size(levels) + int(extra_bytes)
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = self.buf.data_ptr() + off
        betty_reset_status(self)


    @classmethod
    def of_bytes(cls, nbytes: int, device="cuda") -> "Workspace":
        """Scratch for calls that say how much they need themselves (the operators of a residual block)."""
        ws = cls.__new__(cls)
        ws.nbytes = max(int(nbytes), 256)
        ws.buf = torch.empty(ws.nbytes + 256, dtype=torch.uint8, device=device)
        ws.ptr = ws.buf.data_ptr() + (-ws.buf.data_ptr()) % 256
        betty_reset_status(ws)
        return ws


def betty_reset_status(ws: Workspace, stream=None) -> None:
    _check(lib().betty_reset_status(ws.ptr, ws.nbytes, _stream(stream)), "betty_reset_status")


def betty_poll_status(ws: Workspace, stream=None, raise_on_error: bool = True):
    """Synchronises the stream; returns (status, cg_iters)."""
    it = C.c_int32(0)
    st = lib().betty_poll_status(ws.ptr, _stream(stream), C.byref(it))
    if raise_on_error:
        _check(st, "betty_poll_status")
    return st, int(it.value)


def betty_lower_step(L: Level, n_steps: int, ws: Workspace, stream=None) -> None:
    _check(lib().betty_lower_step(L.ref, int(n_steps), ws.ptr, ws.nbytes, _stream(stream)), "betty_lower_step")


def betty_grad(L: Level, wrt: Level, out: torch.Tensor, ws: Workspace, stream=None) -> None:
    _check(lib().betty_grad(L.ref, wrt.ref, _ptr(out), ws.ptr, ws.nbytes, _stream(stream)), "betty_grad")


def betty_hvp(L: Level, u: torch.Tensor, Hu: torch.Tensor, ws: Workspace, stream=None) -> None:
    _check(lib().betty_hvp(L.ref, _ptr(u), _ptr(Hu), ws.ptr, ws.nbytes, _stream(stream)), "betty_hvp")


def betty_mixed_vjp(L: Level, wrt: Level, q: torch.Tensor, out: torch.Tensor, ws: Workspace, stream=None) -> None:
    _check(lib().betty_mixed_vjp(L.ref, wrt.ref, _ptr(q), _ptr(out), ws.ptr, ws.nbytes, _stream(stream)),
           "betty_mixed_vjp")


def betty_hypergrad_neumann(lower: Level, upper: Level, wrt: Level, K: int, alpha: float, out: torch.Tensor,
                            ws: Workspace, stream=None) -> None:
    _check(lib().betty_hypergrad_neumann(lower.ref, upper.ref, wrt.ref, int(K), float(alpha), _ptr(out), ws.ptr,
                                         ws.nbytes, _stream(stream)), "betty_hypergrad_neumann")


def betty_hypergrad_cg(lower: Level, upper: Level, wrt: Level, K: int, tol: float, out: torch.Tensor,
                       ws: Workspace, stream=None) -> None:
    _check(lib().betty_hypergrad_cg(lower.ref, upper.ref, wrt.ref, int(K), float(tol), _ptr(out), ws.ptr, ws.nbytes,
                                    _stream(stream)), "betty_hypergrad_cg")


def betty_hypergrad_fd(lower: Level, upper: Level, wrt: Level, eps0: float, alpha: float, out: torch.Tensor,
                       ws: Workspace, stream=None) -> None:
    _check(lib().betty_hypergrad_fd(lower.ref, upper.ref, wrt.ref, float(eps0), float(alpha), _ptr(out), ws.ptr,
                                    ws.nbytes, _stream(stream)), "betty_hypergrad_fd")


def betty_hypergrad_itd(lower: Level, upper: Level, wrt: Level, n_steps: int, out: torch.Tensor, ws: Workspace,
                        stream=None) -> None:
    _check(lib().betty_hypergrad_itd(lower.ref, upper.ref, wrt.ref, int(n_steps), _ptr(out), ws.ptr, ws.nbytes,
                                     _stream(stream)), "betty_hypergrad_itd")


def betty_chain_levels(levels: Sequence[Level], path: Sequence[int], per_edge: Sequence[MethodCfg],
                       v_in: Optional[torch.Tensor], out: torch.Tensor, accumulate: bool, ws: Workspace,
                       stream=None) -> None:
    arr = _level_array(levels)
    p = (C.c_int32 * len(path))(*[int(i) for i in path])
    cfgs = (_MethodCfg * len(per_edge))(*[m.c for m in per_edge])
    _check(lib().betty_chain_levels(arr, len(levels), p, len(path), cfgs, _ptr(v_in), _ptr(out),
                                    1 if accumulate else 0, ws.ptr, ws.nbytes, _stream(stream)), "betty_chain_levels")


def betty_hvp_logreg_static(X: torch.Tensor, w: torch.Tensor, lam: torch.Tensor, u: torch.Tensor, Hu: torch.Tensor,
                            status_dev: Optional[torch.Tensor] = None, stream=None) -> None:
    """Logistic weight-decay HVP that uses the library's built-in scratch instead of a workspace
    (for callers that cannot allocate device memory); see betty.h for the limits."""
    n, d = X.shape
    _check(lib().betty_hvp_logreg_static(_ptr(X) if n else None, n, d, _ptr(w), _ptr(lam), _ptr(u), _ptr(Hu),
                                         _ptr(status_dev), _stream(stream)), "betty_hvp_logreg_static")


def betty_gemm_bf16(M: int, N: int, pairs, Cout: torch.Tensor, ldc: int, beta: float, path: int, ws: Workspace,
                    stream=None) -> None:
    """pairs: sequence of (A, lda, a_transposed, B, ldb, b_transposed, K, alpha) with bf16 device tensors."""
    arr = (_GemmOperands * len(pairs))()
    for i, (A, lda, ta, B, ldb, tb, K, alpha) in enumerate(pairs):
        arr[i] = _GemmOperands(_ptr(A), int(lda), int(bool(ta)), _ptr(B), int(ldb), int(bool(tb)), int(K), float(alpha))
    _check(lib().betty_gemm_bf16(int(M), int(N), len(pairs), arr, _ptr(Cout), int(ldc), float(beta), int(path), ws.ptr,
                                 ws.nbytes, _stream(stream)), "betty_gemm_bf16")


def _edges(pairs):
    arr = (_Edge * max(1, len(pairs)))()
    for i, (a, b) in enumerate(pairs):
        arr[i] = _Edge(int(a), int(b))
    return arr


def betty_find_paths(n_levels: int, u2l, l2u, k: int, targets) -> list:
    """Valid paths [k, q(1), ..., q(m)] of the dataflow graph (host-only call)."""
    t = (C.c_int32 * max(1, len(targets)))(*[int(x) for x in targets])
    n_paths, n_ints = C.c_int32(0), C.c_int32(0)
    eu, el = _edges(u2l), _edges(l2u)
    _check(lib().betty_find_paths(n_levels, eu, len(u2l), el, len(l2u), int(k), t, len(targets), None, 0,
                                  C.byref(n_paths), C.byref(n_ints)), "betty_find_paths")
    buf = (C.c_int32 * max(1, n_ints.value))()
    _check(lib().betty_find_paths(n_levels, eu, len(u2l), el, len(l2u), int(k), t, len(targets), buf, n_ints.value,
                                  C.byref(n_paths), C.byref(n_ints)), "betty_find_paths")
    out, i = [], 0
    for _ in range(n_paths.value):
        ln = buf[i]
        out.append([buf[i + 1 + j] for j in range(ln)])
        i += 1 + ln
    return out


def betty_hypergrad_graph(levels: Sequence[Level], u2l, l2u, k: int, per_level: Sequence[MethodCfg], out: torch.Tensor,
                          ws: Workspace, stream=None) -> None:
    arr = _level_array(levels)
    cfgs = (_MethodCfg * len(per_level))(*[m.c for m in per_level])
    _check(lib().betty_hypergrad_graph(arr, len(levels), _edges(u2l), len(u2l), _edges(l2u), len(l2u), int(k), cfgs,
                                       _ptr(out), ws.ptr, ws.nbytes, _stream(stream)), "betty_hypergrad_graph")


def betty_engine_run(levels: Sequence[Level], u2l, l2u, per_level: Sequence[MethodCfg], unroll_steps: Sequence[int],
                     n_iterations: int, ws: Workspace, stream=None, log_capacity: int = 65536) -> list:
    """Runs the program's execution schedule (Sec. 3.3); returns the order in which problems stepped."""
    arr = _level_array(levels)
    cfgs = (_MethodCfg * len(per_level))(*[m.c for m in per_level])
    un = (C.c_int32 * len(unroll_steps))(*[int(x) for x in unroll_steps])
    log = (C.c_int32 * log_capacity)()
    n = C.c_int32(0)
    _check(lib().betty_engine_run(arr, len(levels), _edges(u2l), len(u2l), _edges(l2u), len(l2u), cfgs, un,
                                  int(n_iterations), log, log_capacity, C.byref(n), ws.ptr, ws.nbytes, _stream(stream)),
           "betty_engine_run")
    return [log[i] for i in range(min(n.value, log_capacity))]


# ---- operators of a trained residual block ----
def _mat(t: Optional[torch.Tensor], rows: int, cols: int, dtype: torch.dtype, name: str):
    """Address and leading dimension of a [rows, cols] matrix with consecutive values in a row."""
    if t is None:
        return None, 0
    if t.dtype is dtype and t.is_cuda and t.shape == (rows, cols) and t.is_contiguous():
        return t.data_ptr(), cols
    if t.dtype is not dtype or not t.is_cuda:
        raise ValueError(f"{name} must be a {dtype} CUDA tensor, got {t.dtype} on {t.device}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must have the shape ({rows}, {cols}), got {tuple(t.shape)}")
    ld, inner = t.stride()
    if inner != 1 and cols > 1 and rows > 0:
        raise ValueError(f"{name} must have consecutive values in a row, got strides {t.stride()}")
    return t.data_ptr(), ld


_FLOAT = (torch.float32, torch.bfloat16, torch.float16)


def _float_dtype(t: torch.dtype) -> int:
    if t not in _FLOAT:
        raise ValueError(f"fp32, bf16 or fp16 tensors are taken, got {t}")
    return _DT[t]


class BlockNorm:
    """Configuration of betty_block_norm (betty.h): the norms before (`pre`) and after (`post`) a block, its gate and the
    rows that share a gate row.  Parameters are one fp32 tensor [3, d] = (w_pre, w_post, residual scale), with bias
    [5, d] = (..., b_pre, b_post)."""

    def __init__(self, d: int, pre: int = NORM_RMS, post: int = NORM_RMS, gate: int = GATE_NONE, rows_per_gate: int = 1,
                 eps: float = 1e-6, bias: bool = False):
        self.d, self.bias, self.rows_per_gate = int(d), bool(bias), int(rows_per_gate)
        self._fields = (int(pre), int(post), int(gate), int(self.bias), self.rows_per_gate, float(eps))
        self._refs = {}

    def _ref(self, tx: torch.dtype, ty: torch.dtype):
        """The C descriptor for these types (one per pair of types, so that calls of several threads share none in change)."""
        r = self._refs.get((tx, ty))
        if r is None:
            r = self._refs[tx, ty] = C.byref(_BlockNormCfg(self.d, _float_dtype(tx), _float_dtype(ty), *self._fields))
        return r

    def _params(self, t: torch.Tensor, name: str) -> int:
        n = 5 if self.bias else 3
        if t.dtype is not torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n * self.d:
            raise ValueError(f"{name} must be a contiguous fp32 CUDA tensor of {n} x {self.d} values")
        return t.data_ptr()

    def _gate(self, t, rows: int, dtype, name: str):
        return _mat(t, -(-rows // max(self.rows_per_gate, 1)), self.d, dtype, name)


def betty_block_norm(cfg: BlockNorm, params: torch.Tensor, x: torch.Tensor, y: Optional[torch.Tensor], gate: Optional[torch.Tensor],
                     x_out: Optional[torch.Tensor], u: Optional[torch.Tensor], stream=None) -> None:
    """x_out = x + s a(gate) N_post(y), u = N_pre(x_out); y None: u = N_pre(x); u None: no entry norm."""
    rows, d = x.shape[0], cfg.d
    like = y if y is not None else u
    if like is None:
        raise ValueError("one of y and u has to be given")
    tx, ty = x.dtype, like.dtype
    _check(lib().betty_block_norm(cfg._ref(tx, ty), cfg._params(params, "params"), rows, *_mat(x, rows, d, tx, "x"), *_mat(y, rows, d, ty, "y"),
                                  *cfg._gate(gate, rows, ty, "gate"), *_mat(x_out, rows, d, tx, "x_out"), *_mat(u, rows, d, ty, "u"),
                                  _stream(stream)), "betty_block_norm")


def betty_block_norm_workspace_size(cfg: BlockNorm, rows: int, any_layout: bool = True) -> int:
    """any_layout False: for contiguous matrices (and slices of wider ones next to contiguous ones)."""
    out = C.c_size_t(0)
    _check(lib().betty_block_norm_workspace_size_for(cfg._ref(torch.float32, torch.float32), int(rows), int(any_layout), C.byref(out)),
           "betty_block_norm_workspace_size")
    return int(out.value)


def betty_block_norm_backward(cfg: BlockNorm, params: torch.Tensor, x_out: Optional[torch.Tensor], y: Optional[torch.Tensor],
                              gate: Optional[torch.Tensor], du: Optional[torch.Tensor], dx_out: Optional[torch.Tensor],
                              dx: torch.Tensor, dy: Optional[torch.Tensor], dgate: Optional[torch.Tensor], dparams: torch.Tensor,
                              ws: Workspace, stream=None) -> None:
    """Gradients of betty_block_norm from x_out, y and gate; du and dx_out are the gradients of u and x_out."""
    rows, d = dx.shape[0], cfg.d
    like = y if y is not None else du
    if like is None:
        raise ValueError("one of y and du has to be given")
    tx, ty = dx.dtype, like.dtype
    _check(lib().betty_block_norm_backward(
        cfg._ref(tx, ty), cfg._params(params, "params"), rows, *_mat(x_out, rows, d, tx, "x_out"), *_mat(y, rows, d, ty, "y"),
        *cfg._gate(gate, rows, ty, "gate"), *_mat(du, rows, d, ty, "du"), *_mat(dx_out, rows, d, tx, "dx_out"),
        *_mat(dx, rows, d, tx, "dx"), *_mat(dy, rows, d, ty, "dy"), *cfg._gate(dgate, rows, ty, "dgate"),
        cfg._params(dparams, "dparams"), ws.ptr, ws.nbytes, _stream(stream)), "betty_block_norm_backward")


class Act8:
    """Configuration of the betty_act8 calls (betty.h): a hidden layer of `cols` activations, gated when its
    pre-activation is [gate | value], 2 * cols wide."""

    def __init__(self, cols: int, act: int = ACT_GELU, gated: bool = False):
        self.cols, self.gated = int(cols), bool(gated)
        self.width = self.cols * (2 if self.gated else 1)
        self.n_scales = (self.width // max(self.cols, 1)) * -(-self.cols // 128)
        self._fields = (int(act), int(self.gated))
        self._refs = {}

    def _ref(self, t: torch.dtype):
        r = self._refs.get(t)
        if r is None:
            r = self._refs[t] = C.byref(_Act8Cfg(self.cols, _float_dtype(t), *self._fields))
        return r

    def empty(self, rows: int, device="cuda"):
        """An unfilled checkpoint: (q, scales)."""
        return (torch.empty(rows, self.width, dtype=torch.int8, device=device),
                torch.empty(rows, self.n_scales, dtype=torch.float32, device=device))


def betty_act8_store(cfg: Act8, z: torch.Tensor, act: Optional[torch.Tensor], q: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """act = the layer's activation (None: not wanted); (q, scales) = the 8-bit checkpoint of z."""
    rows, t = z.shape[0], z.dtype
    _check(lib().betty_act8_store(cfg._ref(t), rows, *_mat(z, rows, cfg.width, t, "z"), *_mat(act, rows, cfg.cols, t, "act"),
                                  *_mat(q, rows, cfg.width, torch.int8, "q"), *_mat(scales, rows, cfg.n_scales, torch.float32, "scales"),
                                  _stream(stream)), "betty_act8_store")


def betty_act8_restore(cfg: Act8, q: torch.Tensor, scales: torch.Tensor, z: torch.Tensor, stream=None) -> None:
    """z = the values the checkpoint stands for."""
    rows = z.shape[0]
    _check(lib().betty_act8_restore(cfg._ref(z.dtype), rows, *_mat(q, rows, cfg.width, torch.int8, "q"),
                                    *_mat(scales, rows, cfg.n_scales, torch.float32, "scales"), *_mat(z, rows, cfg.width, z.dtype, "z"),
                                    _stream(stream)), "betty_act8_restore")


def betty_act8_backward(cfg: Act8, q: torch.Tensor, scales: torch.Tensor, da: Optional[torch.Tensor], dz: Optional[torch.Tensor],
                        act: Optional[torch.Tensor], stream=None) -> None:
    """dz = the gradient of the pre-activation from da, act = the activation, both at the checkpoint's values."""
    like = dz if dz is not None else act
    if like is None:
        raise ValueError("one of dz and act has to be given")
    rows, t = like.shape[0], like.dtype
    _check(lib().betty_act8_backward(cfg._ref(t), rows, *_mat(q, rows, cfg.width, torch.int8, "q"),
                                     *_mat(scales, rows, cfg.n_scales, torch.float32, "scales"), *_mat(da, rows, cfg.cols, t, "da"),
                                     *_mat(dz, rows, cfg.width, t, "dz"), *_mat(act, rows, cfg.cols, t, "act"), _stream(stream)),
           "betty_act8_backward")


class Grouped:
    """Configuration of the betty_grouped calls (betty.h): `n_groups` experts with matrices [n_out, n_in], operands of
    `dtype` (BETTY_BF16 or BETTY_F16)."""

    def __init__(self, n_groups: int, n_in: int, n_out: int, dtype: int = BETTY_BF16):
        self.n_groups, self.n_in, self.n_out = int(n_groups), int(n_in), int(n_out)
        self.torch_dtype = {BETTY_BF16: torch.bfloat16, BETTY_F16: torch.float16}.get(int(dtype))
        self._ref = C.byref(_GroupedCfg(self.n_groups, int(dtype), self.n_in, self.n_out))

    def _offsets(self, t: torch.Tensor) -> int:
        if t.dtype is not torch.int32 or not t.is_cuda or not t.is_contiguous() or t.numel() != self.n_groups + 1:
            raise ValueError(f"offsets must be {self.n_groups + 1} contiguous int32 values on the GPU")
        return t.data_ptr()

    def _matrices(self, t: torch.Tensor, dtype: torch.dtype, name: str):
        if t.dtype is not dtype or not t.is_cuda:
            raise ValueError(f"{name} must be a {dtype} CUDA tensor, got {t.dtype} on {t.device}")
        if t.dim() != 3 or t.shape[0] != self.n_groups or t.shape[1] != self.n_out or t.shape[2] != self.n_in:
            raise ValueError(f"{name} must have the shape ({self.n_groups}, {self.n_out}, {self.n_in}), got {tuple(t.shape)}")
        gs, ld, inner = t.stride()
        if inner != 1 and self.n_in > 1:
            raise ValueError(f"{name} must have consecutive values in a row, got strides {t.stride()}")
        return t.data_ptr(), ld, gs


def betty_grouped_workspace_size(cfg: Grouped, rows: int, any_layout: Optional[bool] = None) -> int:
    """any_layout: room for aligned copies of the operands; default: where contiguous operands would need them."""
    if any_layout is None:
        any_layout = cfg.n_in % 8 != 0 or cfg.n_out % 8 != 0
    out = C.c_size_t(0)
    _check(lib().betty_grouped_workspace_size(cfg._ref, int(rows), int(any_layout), C.byref(out)), "betty_grouped_workspace_size")
    return int(out.value)


def betty_grouped_forward(cfg: Grouped, offsets: torch.Tensor, x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, ws: Workspace,
                          stream=None) -> None:
    """y[i] = w[e] x[i] for the rows i of expert e."""
    rows, t = x.shape[0], cfg.torch_dtype
    _check(lib().betty_grouped_forward(cfg._ref, rows, cfg._offsets(offsets), *_mat(x, rows, cfg.n_in, t, "x"), *cfg._matrices(w, t, "w"),
                                       *_mat(y, rows, cfg.n_out, y.dtype, "y"), _DT.get(y.dtype, -1), ws.ptr, ws.nbytes, _stream(stream)),
           "betty_grouped_forward")


def betty_grouped_backward_data(cfg: Grouped, offsets: torch.Tensor, dy: torch.Tensor, w: torch.Tensor, dx: torch.Tensor, ws: Workspace,
                                stream=None) -> None:
    """dx[i] = w[e]^T dy[i] for the rows i of expert e."""
    rows, t = dy.shape[0], cfg.torch_dtype
    _check(lib().betty_grouped_backward_data(cfg._ref, rows, cfg._offsets(offsets), *_mat(dy, rows, cfg.n_out, t, "dy"),
                                             *cfg._matrices(w, t, "w"), *_mat(dx, rows, cfg.n_in, dx.dtype, "dx"), _DT.get(dx.dtype, -1),
                                             ws.ptr, ws.nbytes, _stream(stream)), "betty_grouped_backward_data")


def betty_grouped_backward_weight(cfg: Grouped, offsets: torch.Tensor, dy: torch.Tensor, x: torch.Tensor, dw: torch.Tensor, ws: Workspace,
                                  stream=None) -> None:
    """dw[e] = sum over the rows i of expert e of dy[i] x[i]^T."""
    rows, t = dy.shape[0], cfg.torch_dtype
    _check(lib().betty_grouped_backward_weight(cfg._ref, rows, cfg._offsets(offsets), *_mat(dy, rows, cfg.n_out, t, "dy"),
                                               *_mat(x, rows, cfg.n_in, t, "x"), *cfg._matrices(dw, dw.dtype, "dw"), _DT.get(dw.dtype, -1),
                                               ws.ptr, ws.nbytes, _stream(stream)), "betty_grouped_backward_weight")


# ---- losses over a vocabulary ----
_ID = {torch.int32: BETTY_I32, torch.int64: BETTY_I64}


class VocabLoss:
    """Configuration of the betty_vocab calls (betty.h): logits x . w / temperature over `vocab` tokens, operands of `dtype`
    (BETTY_BF16 or BETTY_F16); smoothing and z_loss belong to the cross entropy."""

    def __init__(self, vocab: int, d: int, dtype: int = BETTY_BF16, temperature: float = 1.0, smoothing: float = 0.0, z_loss: float = 0.0):
        self.vocab, self.d = int(vocab), int(d)
        self.torch_dtype = {BETTY_BF16: torch.bfloat16, BETTY_F16: torch.float16}.get(int(dtype))
        self._ref = C.byref(_VocabCfg(self.vocab, self.d, int(dtype), float(temperature), float(smoothing), float(z_loss)))

    def _operands(self, x: torch.Tensor, w: torch.Tensor):
        t = self.torch_dtype
        if t is None:
            raise ValueError("the operands of a vocabulary loss are bf16 or fp16")
        return (self._ref, x.shape[0], *_mat(x, x.shape[0], self.d, t, "x"), *_mat(w, self.vocab, self.d, t, "w"))

    def _entries(self, ids: torch.Tensor, teacher: torch.Tensor, rows: int):
        if ids.dtype not in _ID:
            raise ValueError(f"ids must be int32 or int64, got {ids.dtype}")
        if ids.dim() != 2:
            raise ValueError(f"ids must have the shape ({rows}, entries), got {tuple(ids.shape)}")
        top = ids.shape[1]
        return (top, *_mat(ids, rows, top, ids.dtype, "ids"), _ID[ids.dtype], *_mat(teacher, rows, top, teacher.dtype, "teacher"),
                _float_dtype(teacher.dtype))

    def _results(self, dx: Optional[torch.Tensor], dw: Optional[torch.Tensor], rows: int):
        out = []
        for t, n, name in ((dx, rows, "dx"), (dw, self.vocab, "dw")):
            out += [None, 0, BETTY_F32] if t is None else [*_mat(t, n, self.d, t.dtype, name), _DT.get(t.dtype, -1)]
        return out


def _row_values(t: torch.Tensor, rows: int, name: str, dtype: torch.dtype = torch.float32) -> int:
    """Address of one value per row."""
    if t.dtype is dtype and t.is_cuda and t.shape == (rows,) and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be {rows} contiguous {dtype} values on the GPU, got {t.dtype} of shape {tuple(t.shape)} on {t.device}")


def _tokens(t: torch.Tensor, rows: int):
    """Address and type of the rows' tokens."""
    if t.dtype not in _ID:
        raise ValueError(f"target must be int32 or int64, got {t.dtype}")
    return _row_values(t, rows, "target", t.dtype), _ID[t.dtype]


def _on_current_device(*tensors) -> None:
    """Kernels run on the current device: operands, results and a workspace of another one are refused before anything is launched."""
    here = _raw_device() if _raw_device is not None and torch.cuda.is_initialized() else torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() not in (here, -1):             # -1: not on a GPU, which is refused where its type is
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{here}")


def betty_vocab_workspace_size(cfg: VocabLoss, rows: int, top: int = 0, any_layout: Optional[bool] = None) -> int:
    """Workspace of any of the calls below on up to `rows` rows with `top` entries each (0: cross entropy only).  any_layout: room for
    an aligned copy of w; default: where a contiguous one would need it."""
    out = C.c_size_t(0)
    _check(lib().betty_vocab_workspace_size(cfg._ref, int(rows), int(top), int(cfg.d % 8 != 0 if any_layout is None else any_layout), C.byref(out)),
           "betty_vocab_workspace_size")
    return int(out.value)


def betty_vocab_ce(cfg: VocabLoss, x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, loss: torch.Tensor, lse: torch.Tensor,
                   ws: Workspace, stream=None) -> None:
    """loss, lse [rows] fp32: the rows' cross entropy with `target` (int32 or int64) and the logarithm of its normaliser."""
    rows = x.shape[0]
    _on_current_device(x, w, target, loss, lse, ws.buf)
    _check(lib().betty_vocab_ce(*cfg._operands(x, w), *_tokens(target, rows), _row_values(loss, rows, "loss"),
                                _row_values(lse, rows, "lse"), ws.ptr, ws.nbytes, _stream(stream)), "betty_vocab_ce")


def betty_vocab_ce_backward(cfg: VocabLoss, x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                            dx: Optional[torch.Tensor], dw: Optional[torch.Tensor], ws: Workspace, stream=None) -> None:
    """dx, dw (None: not wanted) = the gradients of sum(dloss * loss)."""
    rows = x.shape[0]
    _on_current_device(x, w, target, lse, dloss, dx, dw, ws.buf)
    _check(lib().betty_vocab_ce_backward(*cfg._operands(x, w), *_tokens(target, rows),
                                         _row_values(lse, rows, "lse"), _row_values(dloss, rows, "dloss"), *cfg._results(dx, dw, rows), ws.ptr,
                                         ws.nbytes, _stream(stream)), "betty_vocab_ce_backward")


def betty_vocab_distill(cfg: VocabLoss, x: torch.Tensor, w: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, loss: torch.Tensor,
                        lse: torch.Tensor, ws: Workspace, stream=None) -> None:
    """loss [rows] = KL(teacher || student) with the teacher's distribution over its entries (ids, teacher) [rows, top]."""
    rows = x.shape[0]
    _on_current_device(x, w, ids, teacher, loss, lse, ws.buf)
    _check(lib().betty_vocab_distill(*cfg._operands(x, w), *cfg._entries(ids, teacher, rows), _row_values(loss, rows, "loss"),
                                     _row_values(lse, rows, "lse"), ws.ptr, ws.nbytes, _stream(stream)), "betty_vocab_distill")


def betty_vocab_distill_backward(cfg: VocabLoss, x: torch.Tensor, w: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor,
                                 dloss: torch.Tensor, dx: Optional[torch.Tensor], dw: Optional[torch.Tensor], ws: Workspace, stream=None) -> None:
    """dx, dw (None: not wanted) = the gradients of sum(dloss * loss)."""
    rows = x.shape[0]
    _on_current_device(x, w, ids, teacher, lse, dloss, dx, dw, ws.buf)
    _check(lib().betty_vocab_distill_backward(*cfg._operands(x, w), *cfg._entries(ids, teacher, rows), _row_values(lse, rows, "lse"),
                                              _row_values(dloss, rows, "dloss"), *cfg._results(dx, dw, rows), ws.ptr, ws.nbytes, _stream(stream)),
           "betty_vocab_distill_backward")


def betty_selftest_wait_timeout(ws: Workspace, stream=None) -> None:
    _check(lib().betty_selftest_wait_timeout(ws.ptr, ws.nbytes, _stream(stream)), "betty_selftest_wait_timeout")


def betty_selftest_smem_limit(reset: bool, device: int, nbytes: int) -> bool:
    """Host-only: would a launch needing `nbytes` of dynamic shared memory on `device` set the limit?"""
    return bool(lib().betty_selftest_smem_limit(1 if reset else 0, int(device), int(nbytes)))
