"""Binding of libmote.so: ctypes, and for the operators that run on a token or a few the extension module _calls (csrc/torch_calls.cpp),
whose calls take less time.  Argument marshalling only: every step runs in the library's kernels.  torch is used for device
memory and streams."""
from __future__ import annotations

import ctypes as C
import importlib
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmote.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2506_14435_b200.build`; "
                      "there is no fallback path")
lib = C.CDLL(_LIB_PATH)


class _Calls:
    """_calls.so, imported when one of the calls that go through it is made first: it fits one version of torch only, and all others do
    without it."""

    def __getattr__(self, name):
        global _calls
        if name.startswith("__"):
            raise AttributeError(name)
        try:
            _calls = importlib.import_module("._calls", __package__)
        except ImportError as e:
            raise ImportError("paper_2506_14435_b200/_calls.so is missing or was built for another torch: build it with "
                              "`python -m paper_2506_14435_b200.build`; there is no fallback path") from e
        return getattr(_calls, name)


_calls = _Calls()

PATH_AUTO, PATH_SIMT, PATH_TENSOR, PATH_STREAM = 0, 1, 2, 3
DTYPE_F32, DTYPE_BF16 = 0, 1


class mote_layer_t(C.Structure):
    _fields_ = [("d", C.c_int32), ("f", C.c_int32), ("E", C.c_int32), ("k", C.c_int32),
                ("norm_topk", C.c_int32), ("path", C.c_int32),
                ("Wr", C.c_void_p), ("router_bias", C.c_void_p),
                ("gate_packed", C.c_void_p), ("up_packed", C.c_void_p), ("down_packed", C.c_void_p),
                ("alpha_gate", C.c_void_p), ("alpha_up", C.c_void_p), ("alpha_down", C.c_void_p),
                ("sh_gate", C.c_void_p), ("sh_up", C.c_void_p), ("sh_down", C.c_void_p),
                ("shared_bits", C.c_int32),
                ("sh_gate_scale", C.c_void_p), ("sh_up_scale", C.c_void_p), ("sh_down_scale", C.c_void_p)]


_LAYER_POINTERS = [n for n, t in mote_layer_t._fields_ if t is C.c_void_p]   # 11 ahead of shared_bits, 3 behind


class mote_router_t(C.Structure):
    _fields_ = [("d", C.c_int32), ("E", C.c_int32), ("k", C.c_int32), ("scoring", C.c_int32), ("n_groups", C.c_int32),
                ("topk_groups", C.c_int32), ("renorm", C.c_int32), ("scale", C.c_float), ("Wr", C.c_void_p),
                ("w_dtype", C.c_int32), ("logit_bias", C.c_void_p), ("select_bias", C.c_void_p), ("packed", C.c_void_p)]


class mote_block_norm_t(C.Structure):
    _fields_ = [("d", C.c_int32), ("eps", C.c_float), ("scale", C.c_float), ("post_norm", C.c_int32),
                ("post_gain", C.c_void_p), ("pre_gain", C.c_void_p), ("res_dtype", C.c_int32), ("gate_cols", C.c_int32),
                ("gate_dtype", C.c_int32), ("gate_sigmoid", C.c_int32), ("gate_tokens", C.c_int64)]


class mote_linear_t(C.Structure):
    _fields_ = [("N", C.c_int64), ("K", C.c_int64), ("W", C.c_void_p), ("bits", C.c_int32), ("w_scale", C.c_void_p),
                ("bias", C.c_void_p), ("act", C.c_int32)]


TAP_FIELDS = ["topk_idx", "topk_w", "offsets", "perm", "qx", "beta_x", "acc_gate", "acc_up", "h_bf16",
              "qh", "beta_h", "acc_down", "y", "shared_out"]


class mote_taps_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in TAP_FIELDS]


lib.mote_status_string.restype = C.c_char_p
lib.mote_status_string.argtypes = [C.c_int]
lib.mote_ternarize_workspace_bytes.restype = C.c_size_t
lib.mote_ternarize_workspace_bytes.argtypes = []
lib.mote_ternarize_pack.restype = C.c_int
lib.mote_ternarize_pack.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_ternarize_pack_static.restype = C.c_int
lib.mote_ternarize_pack_static.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p,
                                           C.c_void_p]
lib.mote_rtn_quant.restype = C.c_int
lib.mote_rtn_quant.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
lib.mote_quant_act.restype = C.c_int
lib.mote_quant_act.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p,
                               C.c_void_p, C.c_void_p]
lib.mote_route_topk.restype = C.c_int
lib.mote_route_topk.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_int, C.c_int,
                                C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
lib.mote_route_stats.restype = C.c_int
lib.mote_route_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
lib.mote_workspace_bytes.restype = C.c_size_t
lib.mote_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64]
lib.mote_layer_workspace_bytes.restype = C.c_size_t
lib.mote_layer_workspace_bytes.argtypes = [C.POINTER(mote_layer_t), C.c_int64]
lib.mote_host_staging_bytes.restype = C.c_size_t
lib.mote_host_staging_bytes.argtypes = [C.c_int, C.c_int64]
lib.mote_moe_forward.restype = C.c_int
lib.mote_moe_forward.argtypes = [C.POINTER(mote_layer_t), C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                 C.POINTER(mote_taps_t), C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_router_pack_bytes.restype = C.c_size_t
lib.mote_router_pack_bytes.argtypes = [C.c_int, C.c_int64, C.c_int]
lib.mote_router_pack.restype = C.c_int
lib.mote_router_pack.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_route_scored.restype = C.c_int
lib.mote_route_scored.argtypes = [C.POINTER(mote_router_t), C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p]
lib.mote_moe_forward_scored.restype = C.c_int
lib.mote_moe_forward_scored.argtypes = [C.POINTER(mote_layer_t), C.POINTER(mote_router_t), C.c_void_p, C.c_void_p, C.c_int64,
                                        C.c_void_p, C.POINTER(mote_taps_t), C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_block_norm.restype = C.c_int
lib.mote_block_norm.argtypes = [C.POINTER(mote_block_norm_t), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                C.c_void_p, C.c_void_p, C.c_void_p]
lib.mote_linear_workspace_bytes.restype = C.c_size_t
lib.mote_linear_workspace_bytes.argtypes = [C.POINTER(mote_linear_t), C.c_int64]
lib.mote_linear.restype = C.c_int
lib.mote_linear.argtypes = [C.POINTER(mote_linear_t), C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int,
                            C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_stack_workspace_bytes.restype = C.c_size_t
lib.mote_stack_workspace_bytes.argtypes = [C.POINTER(mote_layer_t), C.c_int, C.c_int64]
lib.mote_stack_forward.restype = C.c_int
lib.mote_stack_forward.argtypes = [C.POINTER(mote_layer_t), C.c_int, C.c_float, C.c_void_p, C.c_int64, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_rms_norm.restype = C.c_int
lib.mote_rms_norm.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_float, C.c_void_p, C.c_void_p]
lib.mote_moe_forward_host.restype = C.c_int
lib.mote_moe_forward_host.argtypes = [C.POINTER(mote_layer_t), C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_void_p]
lib.mote_moe_forward_profile.restype = C.c_int
lib.mote_moe_forward_profile.argtypes = [C.POINTER(mote_layer_t), C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                         C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_float)]
lib.mote_device_status.restype = C.c_int
lib.mote_device_status.argtypes = [C.c_void_p, C.c_void_p]
lib.mote_selftest_bounded_wait.restype = C.c_int
lib.mote_selftest_bounded_wait.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p]
lib.mote_int8_mma_peak.restype = C.c_int
lib.mote_int8_mma_peak.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.c_void_p]
lib.mote_last_launch_count.restype = C.c_int
lib.mote_last_launch_count.argtypes = []
lib.mote_last_gemm_tile.restype = C.c_int
lib.mote_last_gemm_tile.argtypes = [C.c_int]


class MoteError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib.mote_status_string(status).decode()} (status {status})")


def _check(status: int, where: str):
    if status != 0:
        raise MoteError(status, where)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    # the handle alone: building the Stream object takes about as long as launching a kernel
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _need_cuda(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("expected contiguous CUDA tensors")


def mote_ternarize_pack(W: torch.Tensor):
    """Eq. 7, 9: W[m, n] (fp32 or bf16, CUDA) -> (packed uint8[m, n/4], alpha float32[1])."""
    _need_cuda(W)
    m, n = W.shape
    dt = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}[W.dtype]
    packed = torch.empty((m, max(n // 4, 1)), dtype=torch.uint8, device=W.device)
    alpha = torch.empty(1, dtype=torch.float32, device=W.device)
    ws_bytes = lib.mote_ternarize_workspace_bytes()
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=W.device)
    _check(lib.mote_ternarize_pack(_ptr(W), dt, m, n, _ptr(packed), _ptr(alpha), _ptr(ws), ws_bytes, _stream()),
           "mote_ternarize_pack")
    return packed, alpha


def mote_ternarize_pack_static(W: torch.Tensor, packed: torch.Tensor, alpha: torch.Tensor):
    """mote_ternarize_pack for callers that may not allocate: the caller passes the outputs
    (packed uint8[m, n/4], alpha float32[1]) and the library uses its built-in 2 KiB of device
    scratch, so neither this wrapper nor the call behind it allocates device memory.  At most 2^31
    elements; calls on one device must not overlap (they share the scratch)."""
    _need_cuda(W, packed, alpha)
    m, n = W.shape
    dt = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}[W.dtype]
    if packed.dtype != torch.uint8 or packed.numel() != m * n // 4 or alpha.dtype != torch.float32:
        raise ValueError("packed must be uint8[m, n/4] and alpha float32[1]")
    _check(lib.mote_ternarize_pack_static(_ptr(W), dt, m, n, _ptr(packed), _ptr(alpha), _stream()),
           "mote_ternarize_pack_static")
    return packed, alpha


def mote_rtn_quant(W: torch.Tensor, bits: int):
    """Section 4.3: RTN absmax codes of W[m, n] (fp32 or bf16, CUDA), one scale per row.
    Returns (q, scale float32[m]); q is int8[m, n] for bits = 8 and uint8[m, n/2] for bits = 4."""
    _need_cuda(W)
    m, n = W.shape
    dt = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}[W.dtype]
    if bits == 8:
        q = torch.empty((m, n), dtype=torch.int8, device=W.device)
    else:
        q = torch.empty((m, max(n // 2, 1)), dtype=torch.uint8, device=W.device)
    scale = torch.empty(m, dtype=torch.float32, device=W.device)
    _check(lib.mote_rtn_quant(_ptr(W), dt, m, n, bits, _ptr(q), _ptr(scale), _stream()), "mote_rtn_quant")
    return q, scale


def mote_quant_act(x: torch.Tensor, want_rowsum: bool = True):
    """Eq. 8: x[T, d] bf16 (CUDA; rows may be strided) -> (q int8[T,d], beta f32[T], rowsum i32[T])."""
    if not x.is_cuda or x.dtype != torch.bfloat16 or x.stride(1) != 1:
        raise ValueError("expected a CUDA bf16 matrix with unit inner stride")
    T, d = x.shape
    q = torch.empty((T, d), dtype=torch.int8, device=x.device)
    beta = torch.empty(T, dtype=torch.float32, device=x.device)
    rowsum = torch.empty(T, dtype=torch.int32, device=x.device) if want_rowsum else None
    _check(lib.mote_quant_act(_ptr(x), T, d, x.stride(0) if T > 1 else d, _ptr(q), _ptr(beta), _ptr(rowsum),
                              _stream()), "mote_quant_act")
    return q, beta, rowsum


def mote_route_topk(x, Wr, bias, k: int, norm_topk: int = 1, want_logits: bool = False):
    """Eq. 3: returns (topk_idx int32[T,k], topk_w f32[T,k], logits f32[T,E] or None)."""
    _need_cuda(x, Wr, bias)
    T, d = x.shape
    E = Wr.shape[0]
    idx = torch.empty((T, k), dtype=torch.int32, device=x.device)
    w = torch.empty((T, k), dtype=torch.float32, device=x.device)
    logits = torch.empty((T, E), dtype=torch.float32, device=x.device) if want_logits else None
    _check(lib.mote_route_topk(_ptr(x), T, d, _ptr(Wr), _ptr(bias), E, k, norm_topk, _ptr(idx), _ptr(w),
                               _ptr(logits), _stream()), "mote_route_topk")
    return idx, w, logits


def mote_route_stats(logits: torch.Tensor, topk_idx: torch.Tensor):
    """Eq. 12: (tokens_per_expert int32[E], prob_sum f32[E]) of a routed batch."""
    _need_cuda(logits, topk_idx)
    T, E = logits.shape
    k = topk_idx.shape[1]
    cnt = torch.empty(E, dtype=torch.int32, device=logits.device)
    ps = torch.empty(E, dtype=torch.float32, device=logits.device)
    _check(lib.mote_route_stats(_ptr(logits), _ptr(topk_idx), T, E, k, _ptr(cnt), _ptr(ps), _stream()),
           "mote_route_stats")
    return cnt, ps


_DTYPES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _here(dev: int):
    # the library works on the current device and stream
    if dev != torch.cuda.current_device():
        raise ValueError("expected tensors on the current CUDA device")


def _vector(t, name: str, n: int, dev):
    """An optional [n] float32 weight, and its address."""
    if t is None:
        return None, None
    if t.dtype is not torch.float32 or not t.is_cuda or tuple(t.shape) != (n,) or (dev is not None and t.get_device() != dev):
        raise ValueError(f"{name}: expected float32 [{n}] on the device of the weights")
    t = t.contiguous()
    return t, t.data_ptr()


SCORINGS = {"softmax": 0, "sigmoid": 1}


class MoteRouter:
    """A scored router's weights and options (mote_router_t): Wr[E, d] fp32 or bf16; scoring "softmax" or "sigmoid"; logit_bias and
    select_bias[E] fp32.  Construction runs mote_router_pack; make a new one when Wr has changed."""

    def __init__(self, Wr, k, scoring="softmax", logit_bias=None, select_bias=None, n_groups=1, topk_groups=1, renorm=True, scale=1.0):
        _need_cuda(Wr)
        if Wr.dim() != 2 or Wr.dtype not in _DTYPES:
            raise ValueError("Wr: expected a float32 or bfloat16 matrix")
        if scoring not in SCORINGS:
            raise ValueError(f"scoring: expected one of {sorted(SCORINGS)}")
        self.E, self.d = Wr.shape
        self.k = k
        self.device = Wr.get_device()
        _here(self.device)
        lb, lb_ptr = _vector(logit_bias, "logit_bias", self.E, self.device)
        sb, sb_ptr = _vector(select_bias, "select_bias", self.E, self.device)
        dt = _DTYPES[Wr.dtype]
        need = lib.mote_router_pack_bytes(self.E, self.d, dt)
        if need == 0:
            raise MoteError(2, "mote_router_pack_bytes")
        packed = torch.empty(need, dtype=torch.uint8, device=Wr.device)
        _check(lib.mote_router_pack(_ptr(Wr), dt, self.E, self.d, _ptr(packed), need, _stream()), "mote_router_pack")
        self.tensors = dict(Wr=Wr, logit_bias=lb, select_bias=sb, packed=packed)
        self.struct = mote_router_t(self.d, self.E, k, SCORINGS[scoring], n_groups, topk_groups, int(renorm), scale,
                                    Wr.data_ptr(), dt, lb_ptr, sb_ptr, packed.data_ptr())
        self._address = C.addressof(self.struct)

    def check_device_status(self):
        """Raises MoteError if a bounded device-side wait has run out in a call since this was last asked (the outputs of that call are
        invalid).  Waits for the current stream."""
        _check(lib.mote_device_status(_ptr(self.tensors["packed"]), _stream()), "MoteRouter (device)")


def mote_route_scored(router: MoteRouter, x: torch.Tensor, want_logits: bool = False):
    """x[T, d] bf16 (rows may be strided) -> (topk_idx int32[T, k], topk_w f32[T, k], logits f32[T, E] or None)."""
    r = _calls.route_scored(router._address, router.device, x, want_logits)
    if type(r) is int:
        raise MoteError(r, "mote_route_scored")
    return r


class MoteBlockNorm:
    """The norms around a block (mote_block_norm_t): post_gain, pre_gain [d] fp32 or None; gate_tokens: consecutive tokens that share
    a row of the gate (1: a row each, 0: one row for all)."""

    def __init__(self, d, eps=1e-6, post_norm=False, post_gain=None, pre_gain=None, scale=1.0, gate_sigmoid=False, gate_tokens=1):
        pg, pg_ptr = _vector(post_gain, "post_gain", d, None)
        ng, ng_ptr = _vector(pre_gain, "pre_gain", d, pg.get_device() if pg is not None else None)
        self.device = pg.get_device() if pg is not None else ng.get_device() if ng is not None else None
        self._device = -1 if self.device is None else self.device
        self.tensors = dict(post_gain=pg, pre_gain=ng)
        # the types of the residual and the gate, and the gate's columns, are the call's
        self.struct = mote_block_norm_t(d, eps, scale, int(post_norm), pg_ptr, ng_ptr, DTYPE_BF16, 0, DTYPE_F32, int(gate_sigmoid), gate_tokens)
        self._address = C.addressof(self.struct)


def mote_block_norm(norm: MoteBlockNorm, y: torch.Tensor, residual=None, gate=None, res_out=None, normed_out=None,
                    want_residual: bool = True, want_normed: bool = True):
    """y[T, d] bf16 -> (res_out [T, d] of the residual's type, normed_out [T, d] bf16); either is None where not wanted.  gate:
    [rows, 1] or [rows, d], bf16 or fp32, with rows = ceil(T / gate_tokens).  res_out may be residual, normed_out may be y."""
    r = _calls.block_norm(norm._address, norm._device, y, residual, gate, res_out, normed_out, want_residual, want_normed)
    if type(r) is int:
        raise MoteError(r, "mote_block_norm")
    return r


ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


class MoteLinear:
    """A projection's weights (mote_linear_t): W[N, K] bf16, or the codes of mote_rtn_quant (bits 8: int8[N, K], bits 4:
    uint8[N, K / 2]) with scale[N] fp32; bias[N] fp32 or None; act one of ACTS."""

    def __init__(self, W, bits=16, scale=None, bias=None, act="none"):
        _need_cuda(W)
        if bits not in (16, 8, 4) or W.dim() != 2 or W.dtype is not {16: torch.bfloat16, 8: torch.int8, 4: torch.uint8}[bits]:
            raise ValueError("W: expected bfloat16 [N, K] (bits 16), int8 [N, K] (8) or uint8 [N, K / 2] (4)")
        if act not in ACTS:
            raise ValueError(f"act: expected one of {sorted(ACTS)}")
        if (scale is None) != (bits == 16):
            raise ValueError("scale: expected with codes, and with codes only")
        self.N, self.K, self.bits = W.shape[0], W.shape[1] * (2 if bits == 4 else 1), bits
        self.device = W.get_device()
        sc, sc_ptr = _vector(scale, "scale", self.N, self.device)
        b, b_ptr = _vector(bias, "bias", self.N, self.device)
        self.tensors = dict(W=W, scale=sc, bias=b)
        self.struct = mote_linear_t(self.N, self.K, W.data_ptr(), bits, sc_ptr, b_ptr, ACTS[act])
        self._address = C.addressof(self.struct)
        self._ws = self._small_ws = None     # the smaller one stays: a captured graph may hold its address
        self._ws_T = -1                      # the workspace serves up to this many tokens
        self._ws_address = self._ws_bytes = 0

    @classmethod
    def quantized(cls, W, bits, bias=None, act="none"):
        """Offline step: RTN codes of W[N, K] (fp32 or bf16) by mote_rtn_quant."""
        q, scale = mote_rtn_quant(W, bits)
        return cls(q, bits=bits, scale=scale, bias=bias, act=act)

    def workspace(self, T: int) -> torch.Tensor:
        if T > self._ws_T:
            need = lib.mote_linear_workspace_bytes(C.byref(self.struct), T)
            if need == 0:
                raise MoteError(2, "mote_linear_workspace_bytes")
            if need > self._ws_bytes:        # at most twice: without room for the codes as bf16, and with it
                self._small_ws = self._ws
                self._ws = torch.empty(need, dtype=torch.uint8, device=self.tensors["W"].device)
                self._ws_address, self._ws_bytes = self._ws.data_ptr(), need
            self._ws_T = T
        return self._ws

    def check_device_status(self):
        """Raises MoteError if a bounded device-side wait has run out in the last call (each clears the word; the outputs of that call are
        invalid).  Waits for the current stream."""
        if self._ws is not None:
            _check(lib.mote_device_status(_ptr(self._ws), _stream()), "MoteLinear (device)")


def mote_linear(linear: MoteLinear, x: torch.Tensor, residual=None, out=None, out_dtype=torch.bfloat16):
    """x[T, K] bf16 (rows may be strided) -> act(x W^T + bias) + residual, [T, N] of out_dtype (or out's type); out may be
    residual.  Uses the layer's own workspace: calls of one MoteLinear that can run at the same time need one object each."""
    if len(x) > linear._ws_T:
        linear.workspace(len(x))
    r = _calls.linear(linear._address, linear.device, x, residual, out, out_dtype, linear._ws_address, linear._ws_bytes)
    if type(r) is int:
        raise MoteError(r, "mote_linear")
    return r


class MoteLayer:
    """Device-resident weights of one MoTE layer plus its mote_layer_t."""

    def __init__(self, d, f, E, k, norm_topk, Wr, router_bias, gate_packed, up_packed, down_packed,
                 alpha_gate, alpha_up, alpha_down, sh_gate, sh_up, sh_down, path=PATH_AUTO,
                 shared_bits=16, sh_gate_scale=None, sh_up_scale=None, sh_down_scale=None):
        self.d, self.f, self.E, self.k, self.norm_topk, self.path = d, f, E, k, norm_topk, path
        self.shared_bits = shared_bits
        self.tensors = dict(Wr=Wr, router_bias=router_bias, gate_packed=gate_packed, up_packed=up_packed,
                            down_packed=down_packed, alpha_gate=alpha_gate, alpha_up=alpha_up,
                            alpha_down=alpha_down, sh_gate=sh_gate, sh_up=sh_up, sh_down=sh_down,
                            sh_gate_scale=sh_gate_scale, sh_up_scale=sh_up_scale, sh_down_scale=sh_down_scale)
        _need_cuda(*self.tensors.values())
        self._ws = None

    @classmethod
    def from_master(cls, master: dict, device="cuda", path=PATH_AUTO):
        """Offline step: upload fp32 master weights (numpy, see workloads.synth.master_layer) and
        ternarize every routed matrix on the device with mote_ternarize_pack."""
        d, f, E = master["d"], master["f"], master["E"]
        dev = torch.device(device)
        packed = {}
        alphas = {}
        for name, shape in (("gate", (f, d)), ("up", (f, d)), ("down", (d, f))):
            buf = torch.empty((E, shape[0], shape[1] // 4), dtype=torch.uint8, device=dev)
            al = torch.empty(E, dtype=torch.float32, device=dev)
            for e in range(E):
                W = torch.from_numpy(master["W_" + name][e]).to(dev)
                p, a = mote_ternarize_pack(W)
                buf[e].copy_(p)
                al[e:e + 1].copy_(a)
            packed[name], alphas[name] = buf, al

        def bf16(bits):
            return torch.from_numpy(bits.view("int16")).view(torch.bfloat16).to(dev)

        bias = master.get("router_bias")
        return cls(d, f, E, master["k"], master["norm_topk"], torch.from_numpy(master["Wr"]).to(dev),
                   None if bias is None else torch.from_numpy(bias).to(dev),
                   packed["gate"], packed["up"], packed["down"], alphas["gate"], alphas["up"], alphas["down"],
                   bf16(master["sh_gate"]), bf16(master["sh_up"]), bf16(master["sh_down"]), path=path)

    @classmethod
    def from_device_draws(cls, d, f, E, k, norm_topk, draw, device="cuda", path=PATH_AUTO):
        """Offline step with weights that are already on the device: draw(name, expert) returns
        fp32 CUDA matrices for "gate"/"up"/"down", bf16 ones for "sh_gate"/"sh_up"/"sh_down",
        fp32 "Wr" and "bias" (or None); every routed matrix goes through mote_ternarize_pack."""
        dev = torch.device(device)
        packed, alphas = {}, {}
        for name, shape in (("gate", (f, d)), ("up", (f, d)), ("down", (d, f))):
            buf = torch.empty((E, shape[0], shape[1] // 4), dtype=torch.uint8, device=dev)
            al = torch.empty(E, dtype=torch.float32, device=dev)
            for e in range(E):
                p, a = mote_ternarize_pack(draw(name, e).contiguous())
                buf[e].copy_(p)
                al[e:e + 1].copy_(a)
            packed[name], alphas[name] = buf, al
        return cls(d, f, E, k, norm_topk, draw("Wr").contiguous(), draw("bias"),
                   packed["gate"], packed["up"], packed["down"], alphas["gate"], alphas["up"], alphas["down"],
                   draw("sh_gate").contiguous(), draw("sh_up").contiguous(), draw("sh_down").contiguous(), path=path)

    def quantize_shared(self, bits: int, path=None) -> "MoteLayer":
        """Section 4.3: a layer with the same routed experts whose (bf16) shared expert is replaced
        by its RTN INT8 / INT4 codes (mote_rtn_quant on the device)."""
        if self.shared_bits != 16:
            raise ValueError("the shared expert is quantized already")
        t = dict(self.tensors)
        for name in ("sh_gate", "sh_up", "sh_down"):
            t[name], t[name + "_scale"] = mote_rtn_quant(self.tensors[name], bits)
        return MoteLayer(self.d, self.f, self.E, self.k, self.norm_topk, path=self.path if path is None else path,
                         shared_bits=bits, **t)

    def struct(self) -> mote_layer_t:
        t = self.tensors
        p = [None if t[n] is None else t[n].data_ptr() for n in _LAYER_POINTERS]
        return mote_layer_t(self.d, self.f, self.E, self.k, self.norm_topk, self.path, *p[:11], self.shared_bits, *p[11:])

    def workspace(self, T: int, host_staging: bool = False, struct: mote_layer_t | None = None) -> torch.Tensor:
        """struct: self.struct(), from a caller that has one at hand."""
        need = lib.mote_layer_workspace_bytes(C.byref(self.struct() if struct is None else struct), T)
        if need == 0:
            raise MoteError(2, "mote_layer_workspace_bytes")
        if host_staging:
            need += lib.mote_host_staging_bytes(self.d, T)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.tensors["Wr"].device)
        return self._ws

    def alloc_taps(self, T: int, names=TAP_FIELDS):
        dev = self.tensors["Wr"].device
        P, d, f, E, k = T * self.k, self.d, self.f, self.E, self.k
        spec = dict(topk_idx=((T, k), torch.int32), topk_w=((T, k), torch.float32),
                    offsets=((E + 1,), torch.int32), perm=((P,), torch.int32), qx=((T, d), torch.int8),
                    beta_x=((T,), torch.float32), acc_gate=((P, f), torch.int32), acc_up=((P, f), torch.int32),
                    h_bf16=((P, f), torch.bfloat16), qh=((P, f), torch.int8), beta_h=((P,), torch.float32),
                    acc_down=((P, d), torch.int32), y=((P, d), torch.float32),
                    shared_out=((T, d), torch.float32))
        return {n: torch.zeros(spec[n][0], dtype=spec[n][1], device=dev) for n in names}


def mote_moe_forward(layer: MoteLayer, x: torch.Tensor, residual=None, out=None, taps: dict | None = None):
    """Eq. 2-8 for x[T, d] bf16 (CUDA).  Returns out[T, d] bf16; fills the tensors in `taps`."""
    _need_cuda(x, residual, out)
    T = x.shape[0]
    if out is None:
        out = torch.empty_like(x)
    s = layer.struct()
    ws = layer.workspace(T, struct=s)
    tp = None
    if taps is not None:
        tp = mote_taps_t()
        for n, t in taps.items():
            setattr(tp, n, t.data_ptr())
        tp = C.byref(tp)
    _check(lib.mote_moe_forward(C.byref(s), _ptr(x), _ptr(residual), T, _ptr(out), tp, _ptr(ws), ws.numel(),
                                _stream()), "mote_moe_forward")
    return out


def mote_moe_forward_scored(layer: MoteLayer, router: MoteRouter, x: torch.Tensor, residual=None, out=None, taps: dict | None = None):
    """mote_moe_forward with `router` (mote_route_scored) in the place of the layer's own."""
    for t, name in ((x, "x"), (residual, "residual"), (out, "out")):
        if t is not None and (t.dtype is not torch.bfloat16 or t.dim() != 2 or tuple(t.shape) != (x.shape[0], layer.d)):
            raise ValueError(f"{name}: expected bfloat16 [T, {layer.d}]")
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name}: requires grad, and there is no backward pass; call under torch.no_grad() or with a detached tensor")
    _need_cuda(x, residual, out)
    _here(router.device)
    if any(t is not None and t.get_device() != router.device for t in (x, residual, out, layer.tensors["Wr"])):
        raise ValueError("expected the layer, its router and the tensors on one device")
    T = x.shape[0]
    if out is None:
        out = torch.empty_like(x)
    s = layer.struct()
    ws = layer.workspace(T, struct=s)
    tp = None
    if taps is not None:
        tp = mote_taps_t()
        for n, t in taps.items():
            setattr(tp, n, t.data_ptr())
        tp = C.byref(tp)
    _check(lib.mote_moe_forward_scored(C.byref(s), C.byref(router.struct), _ptr(x), _ptr(residual), T, _ptr(out), tp, _ptr(ws), ws.numel(),
                                       _stream()), "mote_moe_forward_scored")
    return out


def mote_moe_forward_host(layer: MoteLayer, x_host: torch.Tensor, out_host: torch.Tensor, residual_host=None):
    """Same layer with (pinned) host tensors in and out; synchronises the stream."""
    T = x_host.shape[0]
    s = layer.struct()
    ws = layer.workspace(T, host_staging=True, struct=s)
    _check(lib.mote_moe_forward_host(C.byref(s), _ptr(x_host), _ptr(residual_host), T, _ptr(out_host), _ptr(ws),
                                     ws.numel(), _stream()), "mote_moe_forward_host")
    return out_host


class MoteStack:
    """A list of MoteLayer run back to back with the residual between layers (mote_stack_forward)."""

    def __init__(self, layers):
        self.layers = list(layers)
        self._structs = (mote_layer_t * len(self.layers))(*[l.struct() for l in self.layers])
        self._ws = None

    def workspace(self, T: int) -> torch.Tensor:
        need = lib.mote_stack_workspace_bytes(self._structs, len(self.layers), T)
        if need == 0:
            raise MoteError(2, "mote_stack_workspace_bytes")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.layers[0].tensors["Wr"].device)
        return self._ws


def mote_rms_norm(x: torch.Tensor, eps: float = 1e-6, out=None):
    """The LN of Eq. 2 (RMS normalisation, unit gain) of x[T, d] bf16."""
    _need_cuda(x, out)
    if out is None:
        out = torch.empty_like(x)
    _check(lib.mote_rms_norm(_ptr(x), x.shape[0], x.shape[1], eps, _ptr(out), _stream()), "mote_rms_norm")
    return out


def mote_stack_forward(stack: MoteStack, x: torch.Tensor, out=None, layer_inputs=None, rms_eps: float = 1e-6):
    """x[T, d] bf16 -> x_L[T, d] bf16 after all layers (Eq. 1-2 chained, LN = RMS norm; rms_eps = 0
    chains the layers without normalisation); layer_inputs ([L, T, d] bf16) receives the residual
    stream entering every layer."""
    _need_cuda(x, out, layer_inputs)
    T = x.shape[0]
    if out is None:
        out = torch.empty_like(x)
    ws = stack.workspace(T)
    _check(lib.mote_stack_forward(stack._structs, len(stack.layers), rms_eps, _ptr(x), T, _ptr(out), _ptr(layer_inputs),
                                  _ptr(ws), ws.numel(), _stream()), "mote_stack_forward")
    return out


STAGE_NAMES = ["route", "dispatch", "quant_x", "gateup_ternary", "quant_h", "down_ternary", "shared_gateup",
               "shared_down", "combine"]


def mote_moe_forward_profile(layer: MoteLayer, x: torch.Tensor, out=None, residual=None) -> dict:
    """One forward with CUDA events between the stages; returns {stage: milliseconds}."""
    _need_cuda(x, residual, out)
    T = x.shape[0]
    if out is None:
        out = torch.empty_like(x)
    ws = layer.workspace(T)
    s = layer.struct()
    ms = (C.c_float * len(STAGE_NAMES))()
    _check(lib.mote_moe_forward_profile(C.byref(s), _ptr(x), _ptr(residual), T, _ptr(out), _ptr(ws), ws.numel(),
                                        _stream(), ms), "mote_moe_forward_profile")
    return dict(zip(STAGE_NAMES, [float(v) for v in ms]))


def mote_int8_mma_peak(n_batches: int, repeats: int = 5) -> dict:
    """Times the library's MMA-only kernel (mote_int8_mma_peak) with CUDA events on the current
    stream, `repeats` launches back to back after one warm-up: returns {"tops_best", "tops_median",
    "ms" (sorted), "ms_in_order", "ops" (per launch)}."""
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ops = C.c_double(0.0)
    stream = torch.cuda.current_stream()
    evs = [torch.cuda.Event(enable_timing=True) for _ in range(repeats + 2)]
    evs[0].record(stream)
    for i in range(repeats + 1):
        _check(lib.mote_int8_mma_peak(_ptr(ws), n_batches, C.byref(ops), _stream()), "mote_int8_mma_peak")
        evs[i + 1].record(stream)
    torch.cuda.synchronize()
    times = [evs[i].elapsed_time(evs[i + 1]) for i in range(1, repeats + 1)]
    _check(lib.mote_device_status(_ptr(ws), _stream()), "mote_int8_mma_peak (device)")
    in_order = list(times)
    times.sort()
    return {"tops_best": ops.value / (times[0] * 1e-3) / 1e12,
            "tops_median": ops.value / (times[len(times) // 2] * 1e-3) / 1e12, "ms": times,
            "ms_in_order": in_order, "ops": ops.value}
