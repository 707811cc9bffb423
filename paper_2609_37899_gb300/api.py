"""ctypes binding of libsoma.so (the C ABI in include/soma_api.h).

Argument marshalling only: every step of the SPSA path runs in the CUDA
kernels behind the C ABI.  PyTorch supplies device memory and streams.  The
library is loaded on first use; if it is missing this module raises -- there
is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsoma.so")
V = 256

_lock = threading.Lock()
_lib = None

SOMA_OK = 0
STATUS_NAMES = {0: "SOMA_OK", 1: "SOMA_ERR_INVALID_ARG", 2: "SOMA_ERR_UNSUPPORTED",
                3: "SOMA_ERR_WORKSPACE", 4: "SOMA_ERR_CUDA", 5: "SOMA_ERR_TIMEOUT",
                6: "SOMA_ERR_NONFINITE", 7: "SOMA_ERR_BOUNDS"}


class SomaError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {STATUS_NAMES.get(code, code)} ({status_string(code)})")


class soma_dims(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("embed", ctypes.c_int32), ("hidden", ctypes.c_int32)]


TRACE_KINDS = ("gate", "head", "reduce", "update", "prep")
TRACE_FIRST_ORDER = ("linear_ce", "scan", "adamw")


class soma_body_dims(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("width", ctypes.c_int32), ("blocks", ctypes.c_int32)]


class soma_adam_config(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("delta", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("t", ctypes.c_int32)]


class soma_estimate_options(ctypes.Structure):
    _fields_ = [("probe_kind", ctypes.c_int32), ("batch_per_probe", ctypes.c_int32),
                ("summed_loss", ctypes.c_int32)]


class soma_adamw_tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale",
                                               "master")] + \
               [("count", ctypes.c_int64), ("weight_decay", ctypes.c_double)]


class soma_adamw_config(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("seed", ctypes.c_uint64), ("t", ctypes.c_int32),
                ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32)]


class soma_scan_dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("batch", "steps", "dim")]


class soma_scan_strides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("b", "t", "g")]


class soma_linear_ce_dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "vocab", "dim", "h_stride",
                                              "emb_stride")] + [("dtype", ctypes.c_int32)]


DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
PROBE_KINDS = {"dense": 0, "sparse": 1}
MAX_ACCUM = 64


class soma_kernel_times(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 5), ("launches", ctypes.c_int64 * 5)]


class soma_first_order_times(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 3), ("calls", ctypes.c_int64 * 3)]


def _sig(lib, name, res, args):
    f = getattr(lib, name)
    f.restype = res
    f.argtypes = args


def lib():
    """The loaded libsoma.so; raises if it has not been built."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libsoma.so not found at {LIB_PATH}: build it with "
                               "`python -m paper_2609_37899_gb300.build`")
        _lib = _open(LIB_PATH)
        return _lib


def use_library(path: str):
    """Route every call of this module to the library at `path` (for
    instance the checked build, libsoma_checked.so) and return the handle in
    use before, or None; use_library_handle() puts it back."""
    global _lib
    with _lock:
        old = _lib
        _lib = _open(path)
        return old


def use_library_handle(handle):
    global _lib
    with _lock:
        _lib = handle


def _open(path: str):
    """Load one build of the library and declare the C signatures."""
    if True:
        L = ctypes.CDLL(path)
        vp, sz, i32, i64, u64, f32 = (ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int,
                                      ctypes.c_int64, ctypes.c_uint64, ctypes.c_float)
        _sig(L, "soma_param_count", i64, [soma_dims])
        _sig(L, "soma_workspace_bytes", sz, [soma_dims, i32, i32, i32, i32])
        _sig(L, "soma_init_experts", i32, [vp, i32, soma_dims, u64, f32, vp])
        _sig(L, "soma_spsa_step", i32, [vp, i32, soma_dims, i32, f32, f32, u64, u64, vp, i32,
                                        i32, vp, vp, vp, sz, vp])
        _sig(L, "soma_eval_loss", i32, [vp, i32, soma_dims, vp, i32, i32, vp, vp, sz, vp])
        _sig(L, "soma_spsa_update", i32, [vp, i32, soma_dims, i32, f32, u64, u64, vp, vp])
        _sig(L, "soma_get_status", i32, [vp])
        _sig(L, "soma_status_string", ctypes.c_char_p, [i32])
        _sig(L, "soma_trace_enable", i32, [i32])
        _sig(L, "soma_trace_read", i32, [ctypes.POINTER(soma_kernel_times), i32])
        _sig(L, "soma_trace_read_first_order", i32, [ctypes.POINTER(soma_first_order_times), i32])
        _sig(L, "soma_debug_philox", i32, [u64, vp, vp, i32, vp])
        _sig(L, "soma_debug_rademacher", i32, [u64, u64, i32, i32, i64, i64, vp, vp])
        _sig(L, "soma_debug_tc_gemm", i32, [vp, vp, vp, i32, i32, vp])
        _sig(L, "soma_debug_tc_gemm_ts", i32, [vp, vp, vp, i32, i32, vp])
        _sig(L, "soma_spsa_estimate", i32, [vp, i32, soma_dims, i32, i32, f32, u64, u64, vp, i32,
                                            i32, vp, vp, vp, sz, vp])
        _sig(L, "soma_adam_update", i32, [vp, vp, vp, i32, soma_dims, i32, i32, u64,
                                          ctypes.POINTER(ctypes.c_uint64), i32, vp,
                                          soma_adam_config, vp])
        _sig(L, "soma_debug_probe", i32, [u64, u64, i32, i32, i32, i64, i64, vp, vp])
        i32p = ctypes.POINTER(ctypes.c_int32)
        _sig(L, "soma_mixture_workspace_bytes", sz, [soma_dims, i32, i32p, i32, i32, i32])
        _sig(L, "soma_mixture_nll", i32, [vp, i32, soma_dims, vp, i32, i32, i32p, i32, i32, vp,
                                          vp, sz, vp])
        _sig(L, "soma_spsa_estimate_opts", i32, [vp, i32, soma_dims, i32,
                                                 ctypes.POINTER(soma_estimate_options), f32, u64,
                                                 u64, vp, i32, i32, vp, vp, vp, sz, vp])
        _sig(L, "soma_debug_wait_timeout", i32, [ctypes.c_uint32, vp])
        _sig(L, "soma_debug_scan_timeout", i32, [vp, vp, ctypes.c_uint32, vp])
        bd = soma_body_dims
        _sig(L, "soma_body_param_count", i64, [bd])
        _sig(L, "soma_body_workspace_bytes", sz, [bd, i32, i32, i32, i32])
        _sig(L, "soma_body_spsa_estimate", i32, [vp, i32, bd, vp, i32, i32, f32, u64, u64, vp,
                                                 i32, i32, vp, vp, vp, sz, vp])
        _sig(L, "soma_body_spsa_step", i32, [vp, i32, bd, vp, i32, i32, f32, f32, u64, u64, vp,
                                             i32, i32, vp, vp, vp, sz, vp])
        _sig(L, "soma_body_eval_loss", i32, [vp, i32, bd, vp, vp, i32, i32, vp, vp, sz, vp])
        _sig(L, "soma_body_adam_update", i32, [vp, vp, vp, i32, bd, i32, i32, u64,
                                               ctypes.POINTER(ctypes.c_uint64), i32, vp,
                                               soma_adam_config, vp])
        _sig(L, "soma_debug_body_probe", i32, [u64, u64, i32, i32, bd, i32, i64, i64, vp, vp])
        _sig(L, "soma_adamw_step", i32, [ctypes.POINTER(soma_adamw_tensor), i32,
                                         soma_adamw_config, vp, vp])
        sd, ss = soma_scan_dims, soma_scan_strides
        _sig(L, "soma_scan_checkpoint_count", i64, [sd])
        _sig(L, "soma_scan_workspace_bytes", i64, [sd])
        _sig(L, "soma_scan_forward", i32, [vp, ss, i32, sd, vp, vp, vp, vp, ss, vp, vp, vp, sz,
                                           vp])
        _sig(L, "soma_scan_backward", i32, [vp, ss, i32, sd, vp, vp, vp, vp, ss, vp, vp, ss, vp,
                                            vp, sz, vp])
        _sig(L, "soma_scan_step", i32, [vp, ss, i32, i64, i64, vp, vp, ss, vp])
        cd = soma_linear_ce_dims
        _sig(L, "soma_linear_ce_workspace_bytes", sz, [cd, i32])
        _sig(L, "soma_linear_ce_forward", i32, [vp, vp, cd, vp, i64, vp, vp, vp, sz, vp])
        _sig(L, "soma_linear_ce_backward", i32, [vp, vp, cd, vp, i64, vp, vp, vp, i64, vp, i64,
                                                 vp, sz, vp])
        _sig(L, "soma_checked_build", i32, [])
        _sig(L, "soma_debug_check_line", i32, [vp])
        _sig(L, "soma_debug_check_fail", i32, [vp])
        return L


def status_string(code: int) -> str:
    return lib().soma_status_string(code).decode()


def dims(E: int, H: int) -> soma_dims:
    return soma_dims(V, E, H)


def _check(code: int, what: str):
    if code != SOMA_OK:
        raise SomaError(code, what)


# the current stream's handle without a torch.cuda.Stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        if _raw_stream is not None:
            return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t: torch.Tensor, dtype, name: str, numel: int | None = None) -> ctypes.c_void_p:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous CUDA {dtype} tensor")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: expected {numel} elements, got {t.numel()}")
    return ctypes.c_void_p(t.data_ptr())


def param_count(E: int, H: int) -> int:
    return int(lib().soma_param_count(dims(E, H)))


def workspace_bytes(E: int, H: int, n_experts: int, n_pert: int, batch: int, seq_len: int) -> int:
    return int(lib().soma_workspace_bytes(dims(E, H), n_experts, n_pert, batch, seq_len))


def alloc_workspace(E, H, n_experts, n_pert, batch, seq_len, device="cuda") -> torch.Tensor:
    n = workspace_bytes(E, H, n_experts, n_pert, batch, seq_len)
    if n == 0:
        raise ValueError("invalid sizes for the workspace")
    return torch.empty(n, dtype=torch.uint8, device=device)


def init_experts(params: torch.Tensor, E: int, H: int, seed: int, std: float = 0.0, stream=None):
    n_experts = params.shape[0]
    _check(lib().soma_init_experts(_dev(params, torch.float32, "params",
                                        n_experts * param_count(E, H)),
                                   n_experts, dims(E, H), seed, std, _stream(stream)),
           "soma_init_experts")


def spsa_step(params: torch.Tensor, byte_batch: torch.Tensor, E: int, H: int, n_pert: int,
              eps: float, lr: float, seed: int, step: int, losses: torch.Tensor,
              coef: torch.Tensor | None, workspace: torch.Tensor, stream=None):
    """One SPSA step; params [N, P] fp32 updated in place, losses [N, n_pert, 2],
    coef [N, n_pert] or None, byte_batch [N, B, T+1] uint8 (all on the device)."""
    N, B, T1 = byte_batch.shape
    P = param_count(E, H)
    _check(lib().soma_spsa_step(
        _dev(params, torch.float32, "params", N * P), N, dims(E, H), n_pert, eps, lr, seed, step,
        _dev(byte_batch, torch.uint8, "byte_batch"), B, T1 - 1,
        _dev(losses, torch.float32, "losses", N * n_pert * 2),
        _dev(coef, torch.float32, "coef", N * n_pert) if coef is not None else None,
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_spsa_step")


def spsa_estimate(params: torch.Tensor, byte_batch: torch.Tensor, E: int, H: int, n_pert: int,
                  kind: str, eps: float, seed: int, step: int, losses: torch.Tensor,
                  coef: torch.Tensor, workspace: torch.Tensor, stream=None,
                  batch_per_probe: bool = False, summed_loss: bool = False):
    """Losses [N, n_pert, 2] and coefficients [N, n_pert] of one accumulation
    batch with dense or sparse probes; params are read only.  byte_batch is
    [N, B, T+1], or [N, n_pert, B, T+1] with batch_per_probe; summed_loss
    gives every expert the coefficient of the summed loss (control arm)."""
    N = params.shape[0]
    B, T1 = byte_batch.shape[-2], byte_batch.shape[-1]
    if batch_per_probe:
        assert tuple(byte_batch.shape[:2]) == (N, n_pert), "byte_batch [N, n_pert, B, T+1]"
    P = param_count(E, H)
    opts = soma_estimate_options(PROBE_KINDS[kind], int(batch_per_probe), int(summed_loss))
    _check(lib().soma_spsa_estimate_opts(
        _dev(params, torch.float32, "params", N * P), N, dims(E, H), n_pert, ctypes.byref(opts),
        eps, seed, step, _dev(byte_batch, torch.uint8, "byte_batch"), B, T1 - 1,
        _dev(losses, torch.float32, "losses", N * n_pert * 2),
        _dev(coef, torch.float32, "coef", N * n_pert),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_spsa_estimate")


def adam_update(params: torch.Tensor, m: torch.Tensor, v: torch.Tensor, E: int, H: int,
                kind: str, seed: int, steps, coef: torch.Tensor, lr: float, beta1: float,
                beta2: float, delta: float, weight_decay: float, t: int, stream=None):
    """The Adam step of Eq. localspsa; coef [A, N, n_pert], steps: A host ints."""
    A, N, n_pert = coef.shape
    P = param_count(E, H)
    st = (ctypes.c_uint64 * A)(*[int(x) for x in steps])
    cfg = soma_adam_config(lr, beta1, beta2, delta, weight_decay, t)
    _check(lib().soma_adam_update(
        _dev(params, torch.float32, "params", N * P), _dev(m, torch.float32, "m", N * P),
        _dev(v, torch.float32, "v", N * P), N, dims(E, H), n_pert, PROBE_KINDS[kind], seed, st,
        A, _dev(coef, torch.float32, "coef", A * N * n_pert), cfg, _stream(stream)),
        "soma_adam_update")


def _routes(routes):
    import numpy as np
    rt = np.ascontiguousarray(routes, dtype=np.int32)
    assert rt.ndim == 2, "routes [R, k]"
    return rt, rt.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def mixture_workspace_bytes(E: int, H: int, n_experts: int, routes, seq_len: int) -> int:
    rt, ptr = _routes(routes)
    n = int(lib().soma_mixture_workspace_bytes(dims(E, H), n_experts, ptr, rt.shape[0],
                                               rt.shape[1], seq_len))
    if n == 0:
        raise SomaError(1, "soma_mixture_workspace_bytes: invalid sizes or routes")
    return n


def mixture_nll(params: torch.Tensor, requests: torch.Tensor, E: int, H: int, routes, t0: int,
                nll_out: torch.Tensor, workspace: torch.Tensor, stream=None):
    """Routed inference (Eq. main-mixture): nll_out [R, T - t0] for requests
    [R, T+1] (device) and host routes [R, k]."""
    rt, ptr = _routes(routes)
    R, T1 = requests.shape
    N = params.shape[0]
    _check(lib().soma_mixture_nll(
        _dev(params, torch.float32, "params", N * param_count(E, H)), N, dims(E, H),
        _dev(requests, torch.uint8, "requests"), R, T1 - 1, ptr, rt.shape[1], t0,
        _dev(nll_out, torch.float32, "nll_out", R * (T1 - 1 - t0)),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_mixture_nll")


def eval_loss(params: torch.Tensor, byte_batch: torch.Tensor, E: int, H: int,
              loss_out: torch.Tensor, workspace: torch.Tensor, stream=None):
    N, B, T1 = byte_batch.shape
    _check(lib().soma_eval_loss(
        _dev(params, torch.float32, "params", N * param_count(E, H)), N, dims(E, H),
        _dev(byte_batch, torch.uint8, "byte_batch"), B, T1 - 1,
        _dev(loss_out, torch.float32, "loss_out", N),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_eval_loss")


def spsa_update(params: torch.Tensor, E: int, H: int, lr: float, seed: int, step: int,
                coef: torch.Tensor, stream=None):
    N, n_pert = coef.shape
    _check(lib().soma_spsa_update(
        _dev(params, torch.float32, "params", N * param_count(E, H)), N, dims(E, H), n_pert,
        lr, seed, step, _dev(coef, torch.float32, "coef", N * n_pert), _stream(stream)),
        "soma_spsa_update")


def trace_enable(on: bool = True):
    _check(lib().soma_trace_enable(1 if on else 0), "soma_trace_enable")


def trace_read(reset: bool = True) -> dict:
    """{kind: (total_ms, launches)} of the traced launches (waits for them)."""
    t = soma_kernel_times()
    _check(lib().soma_trace_read(ctypes.byref(t), 1 if reset else 0), "soma_trace_read")
    return {k: (t.ms[j], int(t.launches[j])) for j, k in enumerate(TRACE_KINDS)}


def trace_read_first_order(reset: bool = True) -> dict:
    """{kind: (total_ms, calls)} of the traced first-order calls (waits for them)."""
    t = soma_first_order_times()
    _check(lib().soma_trace_read_first_order(ctypes.byref(t), 1 if reset else 0),
           "soma_trace_read_first_order")
    return {k: (t.ms[j], int(t.calls[j])) for j, k in enumerate(TRACE_FIRST_ORDER)}


def get_status(stream=None) -> int:
    return int(lib().soma_get_status(_stream(stream)))


def debug_philox(seed: int, counters: torch.Tensor, stream=None) -> torch.Tensor:
    """Philox4x32-10 words [n, 4] (int32 bit patterns) for counters [n, 4] int32."""
    n = counters.shape[0]
    out = torch.empty_like(counters)
    _check(lib().soma_debug_philox(seed, _dev(counters, torch.int32, "counters"),
                                   _dev(out, torch.int32, "out"), n, _stream(stream)),
           "soma_debug_philox")
    return out


def debug_rademacher(seed: int, step: int, expert: int, probe: int, p0: int, count: int,
                     device="cuda", stream=None) -> torch.Tensor:
    z = torch.empty(count, dtype=torch.int8, device=device)
    _check(lib().soma_debug_rademacher(seed, step, expert, probe, p0, count,
                                       _dev(z, torch.int8, "z"), _stream(stream)),
           "soma_debug_rademacher")
    return z


def debug_probe(seed: int, step: int, expert: int, probe: int, kind: str, p0: int, count: int,
                device="cuda", stream=None) -> torch.Tensor:
    z = torch.empty(count, dtype=torch.int8, device=device)
    _check(lib().soma_debug_probe(seed, step, expert, probe, PROBE_KINDS[kind], p0, count,
                                  _dev(z, torch.int8, "z"), _stream(stream)),
           "soma_debug_probe")
    return z


def debug_wait_timeout(max_polls: int, stream=None):
    """Launch a kernel whose bounded wait runs out (see soma_api.h)."""
    _check(lib().soma_debug_wait_timeout(max_polls, _stream(stream)), "soma_debug_wait_timeout")


def debug_scan_timeout(src: torch.Tensor, max_polls: int, stream=None) -> torch.Tensor:
    """A stage of the recurrence's kernels that is never filled (see soma_api.h): what arrived of
    src fp32 [1024], and the number of stages filled, as one tensor of 1025."""
    out = torch.full((1025,), float("nan"), device=src.device)
    _check(lib().soma_debug_scan_timeout(_dev(src, torch.float32, "src", 1024),
                                         ctypes.c_void_p(out.data_ptr()), max_polls,
                                         _stream(stream)), "soma_debug_scan_timeout")
    return out


def debug_tc_gemm(a: torch.Tensor, b: torch.Tensor, stream=None,
                  a_in_tmem: bool = False) -> torch.Tensor:
    """a [128, K] fp16, b [N, K] fp16 (CUDA) -> a @ b.T [128, N] fp32 on the tensor cores;
    with a_in_tmem, a is staged in tensor memory (soma_debug_tc_gemm_ts)."""
    n, k = b.shape
    d = torch.empty(128, n, dtype=torch.float32, device=a.device)
    name = "soma_debug_tc_gemm_ts" if a_in_tmem else "soma_debug_tc_gemm"
    _check(getattr(lib(), name)(_dev(a, torch.float16, "a", 128 * k),
                                _dev(b, torch.float16, "b", n * k),
                                _dev(d, torch.float32, "d"), n, k, _stream(stream)), name)
    return d


class SomaExperts:
    """N experts' parameters and scratch on the current GPU, stepped by the
    C ABI.  Holds device tensors only; each call is one library call."""

    def __init__(self, n_experts: int, E: int, H: int, n_pert: int, batch: int, seq_len: int,
                 device="cuda"):
        self.N, self.E, self.H = n_experts, E, H
        self.n_pert, self.batch, self.seq_len = n_pert, batch, seq_len
        self.P = param_count(E, H)
        self.params = torch.zeros(n_experts, self.P, dtype=torch.float32, device=device)
        self.workspace = alloc_workspace(E, H, n_experts, n_pert, batch, seq_len, device)
        self.losses = torch.zeros(n_experts, n_pert, 2, dtype=torch.float32, device=device)
        self.coef = torch.zeros(n_experts, n_pert, dtype=torch.float32, device=device)
        self.loss = torch.zeros(n_experts, dtype=torch.float32, device=device)

    def init(self, seed: int, std: float = 0.0, stream=None):
        init_experts(self.params, self.E, self.H, seed, std, stream)

    def step(self, byte_batch: torch.Tensor, eps: float, lr: float, seed: int, step: int,
             stream=None):
        spsa_step(self.params, byte_batch, self.E, self.H, self.n_pert, eps, lr, seed, step,
                  self.losses, self.coef, self.workspace, stream)
        return self.losses, self.coef

    def eval(self, byte_batch: torch.Tensor, stream=None):
        eval_loss(self.params, byte_batch, self.E, self.H, self.loss, self.workspace, stream)
        return self.loss

    def adam_step(self, byte_batches, eps: float, seed: int, steps, t: int, lr: float,
                  beta1: float = 0.9, beta2: float = 0.999, delta: float = 1e-8,
                  weight_decay: float = 1e-4, kind: str = "sparse", stream=None,
                  batch_per_probe: bool = False, summed_loss: bool = False):
        """The paper's optimizer step: one estimate per accumulation batch
        (byte_batches[a] with probe step counter steps[a]), then the Adam
        update with bias correction for update t.  Moments live on this
        object (zeros before the first update)."""
        A = len(byte_batches)
        if getattr(self, "m", None) is None:
            self.m = torch.zeros_like(self.params)
            self.v = torch.zeros_like(self.params)
        if getattr(self, "coef_acc", None) is None or self.coef_acc.shape[0] != A:
            self.coef_acc = torch.zeros(A, self.N, self.n_pert, dtype=torch.float32,
                                        device=self.params.device)
            self.losses_acc = torch.zeros(A, self.N, self.n_pert, 2, dtype=torch.float32,
                                          device=self.params.device)
        for a in range(A):
            spsa_estimate(self.params, byte_batches[a], self.E, self.H, self.n_pert, kind, eps,
                          seed, steps[a], self.losses_acc[a], self.coef_acc[a], self.workspace,
                          stream, batch_per_probe=batch_per_probe, summed_loss=summed_loss)
        adam_update(self.params, self.m, self.v, self.E, self.H, kind, seed, steps, self.coef_acc,
                    lr, beta1, beta2, delta, weight_decay, t, stream)
        return self.losses_acc, self.coef_acc


# ---------------------------------------------------------------------------
# The paper's expert body (Sec. "Model size"): D pre-norm residual blocks of
# width d (bias-free LSTM, GELU MLP of width 4d), gain-only LayerNorm, and a
# frozen tied head E [256, d] shared by every expert.
# ---------------------------------------------------------------------------

def body_dims(d: int = 32, D: int = 2) -> soma_body_dims:
    return soma_body_dims(V, d, D)


def body_param_count(d: int = 32, D: int = 2) -> int:
    return int(lib().soma_body_param_count(body_dims(d, D)))


def body_workspace_bytes(d: int, D: int, n_experts: int, n_pert: int, batch: int,
                         seq_len: int) -> int:
    return int(lib().soma_body_workspace_bytes(body_dims(d, D), n_experts, n_pert, batch,
                                               seq_len))


def body_alloc_workspace(d, D, n_experts, n_pert, batch, seq_len, device="cuda") -> torch.Tensor:
    n = body_workspace_bytes(d, D, n_experts, n_pert, batch, seq_len)
    if n == 0:
        raise ValueError("invalid sizes for the workspace")
    return torch.empty(n, dtype=torch.uint8, device=device)


def body_spsa_estimate(params: torch.Tensor, head: torch.Tensor, byte_batch: torch.Tensor,
                       d: int, D: int, n_pert: int, kind: str, eps: float, seed: int, step: int,
                       losses: torch.Tensor | None, coef: torch.Tensor, workspace: torch.Tensor,
                       stream=None):
    """Losses [N, n_pert, 2] and coefficients [N, n_pert] of the body;
    params [N, M_body] are read only, head [256, d], byte_batch [N, B, T+1]."""
    N, B, T1 = byte_batch.shape
    P = body_param_count(d, D)
    _check(lib().soma_body_spsa_estimate(
        _dev(params, torch.float32, "params", N * P), N, body_dims(d, D),
        _dev(head, torch.float32, "head", V * d), n_pert, PROBE_KINDS[kind], eps, seed, step,
        _dev(byte_batch, torch.uint8, "byte_batch"), B, T1 - 1,
        _dev(losses, torch.float32, "losses", N * n_pert * 2) if losses is not None else None,
        _dev(coef, torch.float32, "coef", N * n_pert),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_body_spsa_estimate")


def body_spsa_step(params: torch.Tensor, head: torch.Tensor, byte_batch: torch.Tensor, d: int,
                   D: int, n_pert: int, kind: str, eps: float, lr: float, seed: int, step: int,
                   losses: torch.Tensor | None, coef: torch.Tensor | None,
                   workspace: torch.Tensor, stream=None):
    """The body's SPSA step: the estimate, then theta -= lr (1/n) sum_i c_i z_i."""
    N, B, T1 = byte_batch.shape
    P = body_param_count(d, D)
    _check(lib().soma_body_spsa_step(
        _dev(params, torch.float32, "params", N * P), N, body_dims(d, D),
        _dev(head, torch.float32, "head", V * d), n_pert, PROBE_KINDS[kind], eps, lr, seed, step,
        _dev(byte_batch, torch.uint8, "byte_batch"), B, T1 - 1,
        _dev(losses, torch.float32, "losses", N * n_pert * 2) if losses is not None else None,
        _dev(coef, torch.float32, "coef", N * n_pert) if coef is not None else None,
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_body_spsa_step")


def body_eval_loss(params: torch.Tensor, head: torch.Tensor, byte_batch: torch.Tensor, d: int,
                   D: int, workspace: torch.Tensor, stream=None) -> torch.Tensor:
    N, B, T1 = byte_batch.shape
    out = torch.empty(N, dtype=torch.float32, device=params.device)
    _check(lib().soma_body_eval_loss(
        _dev(params, torch.float32, "params", N * body_param_count(d, D)), N, body_dims(d, D),
        _dev(head, torch.float32, "head", V * d), _dev(byte_batch, torch.uint8, "byte_batch"),
        B, T1 - 1, _dev(out, torch.float32, "loss"), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), _stream(stream)), "soma_body_eval_loss")
    return out


def body_adam_update(params: torch.Tensor, m: torch.Tensor, v: torch.Tensor, d: int, D: int,
                     kind: str, seed: int, steps, coef: torch.Tensor, lr: float, beta1: float,
                     beta2: float, delta: float, weight_decay: float, t: int, stream=None):
    """Eq. localspsa on the body; coef [A, N, n_pert], steps: A host ints."""
    A, N, n_pert = coef.shape
    P = body_param_count(d, D)
    st = (ctypes.c_uint64 * A)(*[int(x) for x in steps])
    cfg = soma_adam_config(lr, beta1, beta2, delta, weight_decay, t)
    _check(lib().soma_body_adam_update(
        _dev(params, torch.float32, "params", N * P), _dev(m, torch.float32, "m", N * P),
        _dev(v, torch.float32, "v", N * P), N, body_dims(d, D), n_pert, PROBE_KINDS[kind], seed,
        st, A, _dev(coef, torch.float32, "coef", A * N * n_pert), cfg, _stream(stream)),
        "soma_body_adam_update")


def debug_body_probe(seed: int, step: int, expert: int, probe: int, d: int, D: int, kind: str,
                     p0: int, count: int, stream=None) -> torch.Tensor:
    z = torch.zeros(count, dtype=torch.int8, device="cuda")
    _check(lib().soma_debug_body_probe(seed, step, expert, probe, body_dims(d, D),
                                       PROBE_KINDS[kind], p0, count,
                                       _dev(z, torch.int8, "z"), _stream(stream)),
           "soma_debug_body_probe")
    return z


class SomaBodies:
    """N expert bodies of the paper's architecture with their shared frozen
    head, parameters, workspace and Adam moments resident on the device."""

    def __init__(self, n_experts: int, n_pert: int, batch: int, seq_len: int, d: int = 32,
                 D: int = 2, device: str = "cuda"):
        self.N, self.d, self.D, self.n_pert = n_experts, d, D, n_pert
        self.P = body_param_count(d, D)
        if self.P < 0:
            raise ValueError("unsupported body dims")
        self.params = torch.zeros(n_experts, self.P, dtype=torch.float32, device=device)
        self.head = torch.zeros(V, d, dtype=torch.float32, device=device)
        self.m = torch.zeros_like(self.params)
        self.v = torch.zeros_like(self.params)
        self.workspace = body_alloc_workspace(d, D, n_experts, n_pert, batch, seq_len, device)
        self.losses = torch.empty(n_experts, n_pert, 2, dtype=torch.float32, device=device)
        self.coef = torch.empty(n_experts, n_pert, dtype=torch.float32, device=device)

    def step(self, byte_batch, eps, lr, seed, step, kind="sparse", stream=None):
        body_spsa_step(self.params, self.head, byte_batch, self.d, self.D, self.n_pert, kind, eps,
                       lr, seed, step, self.losses, self.coef, self.workspace, stream)
        return self.losses, self.coef

    def eval(self, byte_batch, stream=None):
        return body_eval_loss(self.params, self.head, byte_batch, self.d, self.D, self.workspace,
                              stream)

    def adam_step(self, byte_batches, eps, seed, steps, t, lr, beta1=0.9, beta2=0.999,
                  delta=1e-8, weight_decay=1e-4, kind="sparse", stream=None):
        """Eq. localspsa: one estimate per accumulation batch, then Adam."""
        A = len(byte_batches)
        coef = torch.empty(A, self.N, self.n_pert, dtype=torch.float32, device=self.params.device)
        losses = torch.empty(A, self.N, self.n_pert, 2, dtype=torch.float32,
                             device=self.params.device)
        for a, bx in enumerate(byte_batches):
            body_spsa_estimate(self.params, self.head, bx, self.d, self.D, self.n_pert, kind, eps,
                               seed, steps[a], losses[a], coef[a], self.workspace, stream)
        body_adam_update(self.params, self.m, self.v, self.d, self.D, kind, seed, steps, coef, lr,
                         beta1, beta2, delta, weight_decay, t, stream)
        return losses, coef


# ---------------------------------------------------------------------------
# First-order training: the gated linear recurrence, linear cross entropy,
# AdamW.
# ---------------------------------------------------------------------------

def _rows(t: torch.Tensor, name: str, shape, dtype) -> tuple:
    """(pointer, strides) of a gate or output tensor: any strides but the
    last dimension's, which must be adjacent."""
    if not t.is_cuda or t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected a CUDA {dtype} tensor of shape {tuple(shape)}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return ctypes.c_void_p(t.data_ptr()), t.stride()


def _opt(t, dtype, name, numel):
    return _dev(t, dtype, name, numel) if t is not None else None


def _gate_dtype(gates: torch.Tensor) -> int:
    if gates.dtype not in DTYPES:
        raise ValueError(f"gates: unsupported dtype {gates.dtype}")
    return DTYPES[gates.dtype]


def scan_alloc_checkpoints(batch: int, steps: int, dim: int, device="cuda") -> torch.Tensor:
    n = int(lib().soma_scan_checkpoint_count(soma_scan_dims(batch, steps, dim)))
    if n < 0:
        raise ValueError("invalid sizes for the checkpoints")
    return torch.empty(n, dtype=torch.float32, device=device)


def scan_workspace_bytes(batch: int, steps: int, dim: int) -> int:
    return int(lib().soma_scan_workspace_bytes(soma_scan_dims(batch, steps, dim)))


def _scan_workspace(d: soma_scan_dims, workspace, device, stream):
    """(pointer, bytes, the tensor) of the caller's workspace, or of one from
    torch's allocator where the sizes need any and none is given."""
    if workspace is None:
        n = int(lib().soma_scan_workspace_bytes(d))
        if n <= 0:
            return None, 0, None
        workspace = torch.empty(n, dtype=torch.uint8, device=device)
        if stream is not None:
            # torch's allocator orders it by the current stream: keep it from
            # being handed out again before `stream` is through with it
            stream.wait_stream(torch.cuda.current_stream())
            workspace.record_stream(stream)
    return _dev(workspace, torch.uint8, "workspace"), workspace.numel(), workspace


def scan_forward(gates: torch.Tensor, h: torch.Tensor, c_last: torch.Tensor | None = None,
                 c0: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                 resets: torch.Tensor | None = None, checkpoints: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None, stream=None):
    """The gated linear recurrence over gates [B, T, 4, D] (pre-activations in
    the order i, f, g, o) into h [B, T, D]; c0 and c_last fp32 [B, D], lengths
    int32 [B], resets uint8 [B, T], checkpoints of scan_alloc_checkpoints for
    a scan_backward call, workspace uint8 of scan_workspace_bytes (taken from
    torch's allocator if not given)."""
    B, T, _, D = gates.shape
    dt, d = _gate_dtype(gates), soma_scan_dims(B, T, D)
    gp, gs = _rows(gates, "gates", (B, T, 4, D), gates.dtype)
    hp, hs = _rows(h, "h", (B, T, D), gates.dtype)
    f32 = torch.float32
    wp, wn, _keep = _scan_workspace(d, workspace, gates.device, stream)
    _check(lib().soma_scan_forward(
        gp, soma_scan_strides(*gs[:3]), dt, d, _opt(c0, f32, "c0", B * D),
        _opt(lengths, torch.int32, "lengths", B), _opt(resets, torch.uint8, "resets", B * T), hp,
        soma_scan_strides(hs[0], hs[1], 0), _opt(c_last, f32, "c_last", B * D),
        _opt(checkpoints, f32, "checkpoints", None if checkpoints is None else
             lib().soma_scan_checkpoint_count(d)), wp, wn, _stream(stream)), "soma_scan_forward")


def scan_backward(gates: torch.Tensor, checkpoints: torch.Tensor, dh: torch.Tensor,
                  dgates: torch.Tensor, dc0: torch.Tensor | None = None,
                  dc_last: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                  resets: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                  stream=None):
    """Gradients of scan_forward: dgates [B, T, 4, D] and dc0 [B, D] from dh
    [B, T, D] and dc_last [B, D], with that call's checkpoints."""
    B, T, _, D = gates.shape
    dt, d = _gate_dtype(gates), soma_scan_dims(B, T, D)
    gp, gs = _rows(gates, "gates", (B, T, 4, D), gates.dtype)
    hp, hs = _rows(dh, "dh", (B, T, D), gates.dtype)
    dp, ds = _rows(dgates, "dgates", (B, T, 4, D), gates.dtype)
    f32 = torch.float32
    wp, wn, _keep = _scan_workspace(d, workspace, gates.device, stream)
    _check(lib().soma_scan_backward(
        gp, soma_scan_strides(*gs[:3]), dt, d,
        _dev(checkpoints, f32, "checkpoints", lib().soma_scan_checkpoint_count(d)),
        _opt(lengths, torch.int32, "lengths", B), _opt(resets, torch.uint8, "resets", B * T), hp,
        soma_scan_strides(hs[0], hs[1], 0), _opt(dc_last, f32, "dc_last", B * D), dp,
        soma_scan_strides(*ds[:3]), _opt(dc0, f32, "dc0", B * D), wp, wn, _stream(stream)),
        "soma_scan_backward")


def scan_step(gates: torch.Tensor, c: torch.Tensor, h: torch.Tensor, stream=None):
    """One token: gates [B, 4, D], state c [B, D] fp32 (updated), h [B, D]."""
    B, _, D = gates.shape
    dt = _gate_dtype(gates)
    gp, gs = _rows(gates, "gates", (B, 4, D), gates.dtype)
    hp, hs = _rows(h, "h", (B, D), gates.dtype)
    _check(lib().soma_scan_step(gp, soma_scan_strides(gs[0], 0, gs[1]), dt, B, D,
                                _dev(c, torch.float32, "c", B * D), hp,
                                soma_scan_strides(hs[0], 0, 0), _stream(stream)),
           "soma_scan_step")


def _row_stride(t: torch.Tensor) -> int:
    """Elements between rows; what the stride of fewer than two rows says does not matter."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _ce_dims(h: torch.Tensor, emb: torch.Tensor) -> soma_linear_ce_dims:
    return soma_linear_ce_dims(h.shape[0], emb.shape[0], h.shape[1], _row_stride(h),
                               _row_stride(emb), DTYPES.get(h.dtype, -1))


def linear_ce_workspace_bytes(rows: int, vocab: int, dim: int, dtype: torch.dtype,
                              backward: bool = True, h_stride: int | None = None,
                              emb_stride: int | None = None) -> int:
    """Bytes that linear_ce_forward needs, and linear_ce_backward with `backward`."""
    d = soma_linear_ce_dims(rows, vocab, dim, h_stride or dim, emb_stride or dim,
                            DTYPES.get(dtype, -1))
    return max(int(lib().soma_linear_ce_workspace_bytes(d, k)) for k in range(1 + bool(backward)))


def linear_ce_alloc_workspace(rows, vocab, dim, dtype, backward=True, h_stride=None,
                              emb_stride=None, device="cuda") -> torch.Tensor:
    n = linear_ce_workspace_bytes(rows, vocab, dim, dtype, backward, h_stride, emb_stride)
    if n == 0:
        raise ValueError("invalid sizes or dtype for the workspace")
    return torch.empty(n, dtype=torch.uint8, device=device)


def linear_ce_forward(h: torch.Tensor, emb: torch.Tensor, targets: torch.Tensor,
                      loss: torch.Tensor, lse: torch.Tensor, workspace: torch.Tensor,
                      ignore_index: int = -100, stream=None):
    """Cross entropy of the head emb [V, d] on states h [N, d] (bf16 or fp16)
    for targets [N] int64: loss and lse [N] fp32, per row."""
    N = h.shape[0]
    hp, _ = _rows(h, "h", (N, emb.shape[1]), emb.dtype)
    ep, _ = _rows(emb, "emb", emb.shape, h.dtype)
    _check(lib().soma_linear_ce_forward(
        hp, ep, _ce_dims(h, emb), _dev(targets, torch.int64, "targets", N), ignore_index,
        _dev(loss, torch.float32, "loss", N), _dev(lse, torch.float32, "lse", N),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
        "soma_linear_ce_forward")


def linear_ce_backward(h: torch.Tensor, emb: torch.Tensor, targets: torch.Tensor,
                       lse: torch.Tensor, dloss: torch.Tensor, dh: torch.Tensor,
                       demb: torch.Tensor, workspace: torch.Tensor, ignore_index: int = -100,
                       stream=None):
    """Gradients of linear_ce_forward: dh [N, d] and demb [V, d] from its lse
    and the gradient dloss [N] fp32 of its losses."""
    N = h.shape[0]
    hp, _ = _rows(h, "h", (N, emb.shape[1]), emb.dtype)
    ep, _ = _rows(emb, "emb", emb.shape, h.dtype)
    dhp, _ = _rows(dh, "dh", h.shape, h.dtype)
    dep, _ = _rows(demb, "demb", emb.shape, h.dtype)
    _check(lib().soma_linear_ce_backward(
        hp, ep, _ce_dims(h, emb), _dev(targets, torch.int64, "targets", N), ignore_index,
        _dev(lse, torch.float32, "lse", N), _dev(dloss, torch.float32, "dloss", N), dhp,
        _row_stride(dh), dep, _row_stride(demb), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), _stream(stream)), "soma_linear_ce_backward")


class AdamW:
    """AdamW over a list of tensors, one library call per step.

    params: contiguous CUDA tensors of one dtype (fp32, bf16 or fp16).
    exp_avg, exp_avg_sq: their moments.  fp32 tensors, or float8_e4m3fn ones
    with the fp32 scales m_scales, v_scales (one per 256 elements); in 8 bits
    exp_avg_sq holds the root of the second moment.  masters: fp32 copies of
    16-bit params, or None.  weight_decay: one value, or one per tensor.
    ``AdamW.zero_state(params, bits)`` makes the moments.  The object keeps
    the tensors and their table; gradients are passed to every step."""

    def __init__(self, params, exp_avg, exp_avg_sq, m_scales=None, v_scales=None, masters=None,
                 weight_decay=0.0):
        n = len(params)
        for name, ts in (("exp_avg", exp_avg), ("exp_avg_sq", exp_avg_sq), ("m_scales", m_scales),
                         ("v_scales", v_scales), ("masters", masters)):
            if ts is not None and len(ts) != n:
                raise ValueError(f"{name}: expected {n} tensors, got {len(ts)}")
        self.param_dtype = params[0].dtype if n else torch.float32
        if self.param_dtype not in DTYPES:
            raise ValueError(f"params: unsupported dtype {self.param_dtype}")
        self.bits = 32 if m_scales is None else 8
        if (m_scales is None) != (v_scales is None):
            raise ValueError("m_scales and v_scales go together")
        state = torch.float32 if self.bits == 32 else torch.float8_e4m3fn
        decay = [float(weight_decay)] * n if not hasattr(weight_decay, "__len__") else weight_decay
        if len(decay) != n:
            raise ValueError(f"weight_decay: expected {n} values, got {len(decay)}")
        self.tensors = (list(params), list(exp_avg), list(exp_avg_sq), m_scales, v_scales, masters)
        self._table = (soma_adamw_tensor * max(n, 1))()
        for k, p in enumerate(params):
            row, size, blocks = self._table[k], p.numel(), -(-p.numel() // 256)
            row.param = _dev(p, self.param_dtype, f"params[{k}]").value
            row.m = _dev(exp_avg[k], state, f"exp_avg[{k}]", size).value
            row.v = _dev(exp_avg_sq[k], state, f"exp_avg_sq[{k}]", size).value
            if self.bits == 8:
                row.m_scale = _dev(m_scales[k], torch.float32, f"m_scales[{k}]", blocks).value
                row.v_scale = _dev(v_scales[k], torch.float32, f"v_scales[{k}]", blocks).value
            if masters is not None:
                row.master = _dev(masters[k], torch.float32, f"masters[{k}]", size).value
            row.count, row.weight_decay = size, float(decay[k])
        self._sizes = [p.numel() for p in params]
        self._addresses = [p.data_ptr() for p in params]
        self._in_table = [0] * n  # the gradients' addresses in the table

    @staticmethod
    def zero_state(params, bits: int = 32) -> dict:
        """Zero moments as keyword arguments of the constructor."""
        if bits == 32:
            return {k: [torch.zeros_like(p, dtype=torch.float32) for p in params]
                    for k in ("exp_avg", "exp_avg_sq")}
        state = {k: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device)
                     .view(torch.float8_e4m3fn) for p in params]
                 for k in ("exp_avg", "exp_avg_sq")}
        return {**state, **{k: [torch.zeros(-(-p.numel() // 256), device=p.device)
                                for p in params] for k in ("m_scales", "v_scales")}}

    def step(self, grads, t: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
             eps: float = 1e-8, seed: int = 0, grad_scale: torch.Tensor | None = None,
             stream=None):
        """Update t (1-based) from grads (one per tensor, one dtype);
        grad_scale: a device fp32 scalar the gradients are multiplied by."""
        params = self.tensors[0]
        if len(grads) != len(params):
            raise ValueError(f"grads: expected {len(params)} tensors, got {len(grads)}")
        dtype = grads[0].dtype if grads else torch.float32
        if dtype not in DTYPES:
            raise ValueError(f"grads: unsupported dtype {dtype}")
        if [p.data_ptr() for p in params] != self._addresses:
            raise ValueError("params were given other memory since the table was made")
        for k, (g, size) in enumerate(zip(grads, self._sizes)):
            if not g.is_cuda or g.dtype != dtype or g.numel() != size or not g.is_contiguous():
                _dev(g, dtype, f"grads[{k}]", size)  # says which it is
            at = g.data_ptr()
            if at != self._in_table[k]:
                self._table[k].grad = self._in_table[k] = at
        cfg = soma_adamw_config(lr, beta1, beta2, eps, seed & (2 ** 64 - 1), t,
                                DTYPES[self.param_dtype], DTYPES[dtype], self.bits)
        _check(lib().soma_adamw_step(
            self._table, len(params), cfg,
            _dev(grad_scale, torch.float32, "grad_scale", 1) if grad_scale is not None else None,
            _stream(stream)), "soma_adamw_step")
