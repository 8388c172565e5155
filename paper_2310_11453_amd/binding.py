"""Thin ctypes binding of libbitlinear.so (see include/bitlinear.h).

Argument marshalling only: every step of BitLinear runs in the HIP kernels.
PyTorch supplies device memory and the current stream, nothing else.  There is
no CPU fallback: a missing library or a missing GPU raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libbitlinear.so"

BL_OK = 0
GAMMA_PER_TOKEN, GAMMA_PER_TENSOR = 0, 1
FLAG_SKIP_LN, FLAG_OUT_ACC_I32, FLAG_BETA_CENTERED = 1, 2, 4
OP_PACK, OP_QUANT, OP_FORWARD, OP_BACKWARD, OP_LN_BACKWARD, OP_FORWARD_NONNEG = 0, 1, 2, 3, 4, 5
OP_MATMUL, OP_ROUTE, OP_QUANT_NONLINEAR = 6, 7, 8
FUNCTIONS = {"relu": 0, "relu2": 1, "gelu": 2, "silu": 3, "relu_marked": 8}
F32, BF16 = 0, 1

EXPORTS = (
    "bitlinear_packed_bytes", "bitlinear_workspace_bytes", "bitlinear_pack_weights",
    "bitlinear_packed_to_canonical", "bitlinear_quant_act", "bitlinear_matmul",
    "bitlinear_forward", "bitlinear_backward_ste", "bitlinear_status_string",
    "bitlinear_packed_bytes_grouped", "bitlinear_workspace_bytes_grouped",
    "bitlinear_pack_weights_grouped", "bitlinear_packed_to_canonical_grouped",
    "bitlinear_quant_act_grouped", "bitlinear_forward_grouped", "bitlinear_layernorm_backward",
    "bitlinear_weight_rowsums", "bitlinear_quant_act_nonneg", "bitlinear_matmul_nonneg",
    "bitlinear_forward_nonneg", "bitlinear_forward_workspace_layout", "bitlinear_set_tuning",
    "bitlinear_forward_static", "bitlinear_probe_read", "bitlinear_weight_rowsums_grouped",
    "bitlinear_quant_act_grouped_nonneg", "bitlinear_forward_grouped_nonneg",
    "bitlinear_workspace_bytes_experts", "bitlinear_route", "bitlinear_matmul_experts",
    "bitlinear_backward_ste_experts", "bitlinear_combine", "bitlinear_combine_backward",
    "bitlinear_quant_nonlinear", "bitlinear_nonlinear_backward",
)

_lib = None


class BitLinearError(RuntimeError):
    pass


def load_library() -> ctypes.CDLL:
    """Loads the in-tree library (build it first: python -m paper_2310_11453_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise BitLinearError(f"{LIB_PATH} is missing: run `python -m paper_2310_11453_amd.build`")
    lib = ctypes.CDLL(str(LIB_PATH))
    i64, u32, vp, sz, ci, cf = (ctypes.c_int64, ctypes.c_uint, ctypes.c_void_p, ctypes.c_size_t,
                                ctypes.c_int, ctypes.c_float)
    lib.bitlinear_packed_bytes.restype = sz
    lib.bitlinear_packed_bytes.argtypes = [i64, i64, u32]
    lib.bitlinear_workspace_bytes.restype = sz
    lib.bitlinear_workspace_bytes.argtypes = [ci, i64, i64, i64, ci, u32]
    lib.bitlinear_pack_weights.restype = ci
    lib.bitlinear_pack_weights.argtypes = [vp, i64, i64, u32, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_packed_to_canonical.restype = ci
    lib.bitlinear_packed_to_canonical.argtypes = [vp, i64, i64, vp, vp]
    lib.bitlinear_quant_act.restype = ci
    lib.bitlinear_quant_act.argtypes = [vp, i64, i64, vp, vp, cf, ci, u32, vp, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_matmul.restype = ci
    lib.bitlinear_matmul.argtypes = [vp, vp, vp, i64, i64, vp, i64, vp, ci, u32, vp, vp, sz, vp]
    lib.bitlinear_forward.restype = ci
    lib.bitlinear_forward.argtypes = [vp, i64, i64, vp, i64, vp, vp, vp, cf, ci, u32, vp, vp, sz, vp]
    lib.bitlinear_backward_ste.restype = ci
    lib.bitlinear_backward_ste.argtypes = [vp, i64, i64, i64, vp, vp, ci, vp, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_packed_bytes_grouped.restype = sz
    lib.bitlinear_packed_bytes_grouped.argtypes = [i64, i64, ci, ci]
    lib.bitlinear_workspace_bytes_grouped.restype = sz
    lib.bitlinear_workspace_bytes_grouped.argtypes = [ci, i64, i64, i64, ci, ci, ci]
    lib.bitlinear_pack_weights_grouped.restype = ci
    lib.bitlinear_pack_weights_grouped.argtypes = [vp, i64, i64, ci, ci, u32, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_packed_to_canonical_grouped.restype = ci
    lib.bitlinear_packed_to_canonical_grouped.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.bitlinear_quant_act_grouped.restype = ci
    lib.bitlinear_quant_act_grouped.argtypes = [vp, i64, i64, ci, vp, vp, cf, ci, u32, vp, vp, vp, vp,
                                                vp, sz, vp]
    lib.bitlinear_forward_grouped.restype = ci
    lib.bitlinear_forward_grouped.argtypes = [vp, i64, i64, vp, i64, ci, ci, vp, vp, vp, cf, ci, u32,
                                              vp, vp, sz, vp]
    lib.bitlinear_layernorm_backward.restype = ci
    lib.bitlinear_layernorm_backward.argtypes = [vp, vp, i64, i64, ci, vp, cf, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_weight_rowsums.restype = ci
    lib.bitlinear_weight_rowsums.argtypes = [vp, i64, i64, vp, vp]
    lib.bitlinear_quant_act_nonneg.restype = ci
    lib.bitlinear_quant_act_nonneg.argtypes = [vp, i64, i64, vp, vp, cf, ci, u32, vp, vp, vp, vp, vp,
                                               vp, sz, vp]
    lib.bitlinear_matmul_nonneg.restype = ci
    lib.bitlinear_matmul_nonneg.argtypes = [vp, vp, vp, vp, i64, i64, vp, i64, vp, vp, ci, u32, vp, vp]
    lib.bitlinear_forward_nonneg.restype = ci
    lib.bitlinear_forward_nonneg.argtypes = [vp, i64, i64, vp, i64, vp, vp, vp, vp, cf, ci, u32, vp,
                                             vp, sz, vp]
    lib.bitlinear_forward_static.restype = ci
    lib.bitlinear_forward_static.argtypes = [vp, i64, i64, vp, i64, vp, vp, vp, cf, ci, u32, vp, vp]
    lib.bitlinear_weight_rowsums_grouped.restype = ci
    lib.bitlinear_weight_rowsums_grouped.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.bitlinear_quant_act_grouped_nonneg.restype = ci
    lib.bitlinear_quant_act_grouped_nonneg.argtypes = [vp, i64, i64, ci, vp, vp, cf, ci, u32, vp, vp, vp,
                                                       vp, vp, vp, sz, vp]
    lib.bitlinear_forward_grouped_nonneg.restype = ci
    lib.bitlinear_forward_grouped_nonneg.argtypes = [vp, i64, i64, vp, i64, ci, ci, vp, vp, vp, vp, cf,
                                                     ci, u32, vp, vp, sz, vp]
    lib.bitlinear_workspace_bytes_experts.restype = sz
    lib.bitlinear_workspace_bytes_experts.argtypes = [ci, i64, ci, i64, i64, ci, ci]
    lib.bitlinear_route.restype = ci
    lib.bitlinear_route.argtypes = [vp, i64, ci, ci, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_matmul_experts.restype = ci
    lib.bitlinear_matmul_experts.argtypes = [vp, vp, vp, i64, ci, i64, vp, vp, ci, vp, i64, vp, ci, u32, vp, vp]
    lib.bitlinear_backward_ste_experts.restype = ci
    lib.bitlinear_backward_ste_experts.argtypes = [vp, i64, ci, i64, i64, vp, vp, ci, vp, vp, ci, vp, vp, vp, vp,
                                                   vp, sz, vp]
    lib.bitlinear_combine.restype = ci
    lib.bitlinear_combine.argtypes = [vp, vp, vp, i64, ci, i64, vp, vp]
    lib.bitlinear_combine_backward.restype = ci
    lib.bitlinear_combine_backward.argtypes = [vp, vp, vp, vp, i64, ci, i64, vp, vp, vp]
    lib.bitlinear_quant_nonlinear.restype = ci
    lib.bitlinear_quant_nonlinear.argtypes = [vp, i64, i64, ci, cf, vp, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.bitlinear_nonlinear_backward.restype = ci
    lib.bitlinear_nonlinear_backward.argtypes = [vp, vp, vp, i64, i64, ci, cf, vp, ci, vp, vp]
    lib.bitlinear_probe_read.restype = ci
    lib.bitlinear_probe_read.argtypes = [vp, sz, ci, ci, vp, vp]
    lib.bitlinear_forward_workspace_layout.restype = ci
    lib.bitlinear_forward_workspace_layout.argtypes = [i64, i64, i64, ci, ctypes.POINTER(sz)]
    lib.bitlinear_set_tuning.restype = ci
    lib.bitlinear_set_tuning.argtypes = [ctypes.c_char_p]
    lib.bitlinear_status_string.restype = ctypes.c_char_p
    lib.bitlinear_status_string.argtypes = [ci]
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().bitlinear_status_string(code).decode()


def _check(code: int, what: str) -> None:
    if code != BL_OK:
        raise BitLinearError(f"{what}: {status_string(code)} ({code})")


def _ptr(t: torch.Tensor | None, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise BitLinearError("tensor is not on the GPU")
    if not t.is_contiguous():
        raise BitLinearError("tensor is not contiguous")
    if dtype is not None and t.dtype != dtype:
        raise BitLinearError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream():
    # the current stream of the current device; building a torch.cuda.Stream object for it costs 2.6 us
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _gran(per_tensor: bool) -> int:
    return GAMMA_PER_TENSOR if per_tensor else GAMMA_PER_TOKEN


def packed_bytes(N: int, K: int, flags: int = 0) -> int:
    return int(load_library().bitlinear_packed_bytes(N, K, flags))


def workspace_bytes(op: int, M: int, N: int, K: int, per_tensor: bool = False, flags: int = 0) -> int:
    return int(load_library().bitlinear_workspace_bytes(op, M, N, K, _gran(per_tensor), flags))


def set_tuning(spec: str | None = None) -> None:
    """Launch-time switches for tests and benchmarks ("name=value,..."; None resets)."""
    _check(load_library().bitlinear_set_tuning(None if spec is None else spec.encode()),
           "bitlinear_set_tuning")


def forward_workspace_layout(M: int, N: int, K: int, per_tensor: bool = False) -> dict:
    """Byte offsets of what bitlinear_forward leaves in its workspace (xhat: M = 1 only)."""
    off = (ctypes.c_size_t * 4)()
    _check(load_library().bitlinear_forward_workspace_layout(M, N, K, _gran(per_tensor), off),
           "bitlinear_forward_workspace_layout")
    return dict(codes=off[0], gamma=off[1], rowsum=off[2],
                xhat=None if off[3] == ctypes.c_size_t(-1).value else off[3])


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def bitlinear_pack_weights(W: torch.Tensor, flags: int = 0, workspace: torch.Tensor | None = None):
    """Eq. 1-3, 12.  Returns (packed uint8 blob, alpha [1], beta [1]) on W's device."""
    lib = load_library()
    N, K = W.shape
    nbytes = packed_bytes(N, K, flags)
    if nbytes == 0:
        _check(-2, "bitlinear_pack_weights")
    packed = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    alpha = torch.empty(1, dtype=torch.float32, device=W.device)
    beta = torch.empty(1, dtype=torch.float32, device=W.device)
    ws = workspace if workspace is not None else _workspace(workspace_bytes(OP_PACK, 0, N, K), W.device)
    _check(lib.bitlinear_pack_weights(_ptr(W, torch.float32), N, K, flags, _ptr(packed), _ptr(alpha),
                                      _ptr(beta), _ptr(ws), ws.numel(), _stream()),
           "bitlinear_pack_weights")
    return packed, alpha, beta


def bitlinear_packed_to_canonical(packed: torch.Tensor, N: int, K: int) -> torch.Tensor:
    """Blob -> int32 tensor [N, K/32] holding the canonical uint32 words."""
    out = torch.empty((N, K // 32), dtype=torch.int32, device=packed.device)
    _check(load_library().bitlinear_packed_to_canonical(_ptr(packed), N, K, _ptr(out), _stream()),
           "bitlinear_packed_to_canonical")
    return out


def bitlinear_quant_act(X: torch.Tensor, ln_eps: float = 1e-5, per_tensor: bool = False,
                        flags: int = 0, ln_gain=None, ln_bias=None, want_xhat: bool = False,
                        workspace: torch.Tensor | None = None):
    """Eq. 12 + Eq. 4-5.  Returns (codes int8 [M,K], gamma, rowsum int32 [M], xhat or None)."""
    M, K = X.shape
    dev = X.device
    codes = torch.empty((M, K), dtype=torch.int8, device=dev)
    gamma = torch.empty(1 if per_tensor else max(M, 1), dtype=torch.float32, device=dev)
    rowsum = torch.empty(max(M, 1), dtype=torch.int32, device=dev)
    xhat = torch.empty((M, K), dtype=torch.float32, device=dev) if want_xhat else None
    ws = workspace if workspace is not None else _workspace(
        workspace_bytes(OP_QUANT, M, 1, K, per_tensor), dev)
    _check(load_library().bitlinear_quant_act(
        _ptr(X, torch.float32), M, K, _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32),
        ln_eps, _gran(per_tensor), flags, _ptr(codes), _ptr(gamma), _ptr(rowsum), _ptr(xhat),
        _ptr(ws), ws.numel(), _stream()), "bitlinear_quant_act")
    return codes, gamma, rowsum, xhat


def bitlinear_matmul(codes: torch.Tensor, gamma: torch.Tensor, rowsum: torch.Tensor,
                     packed: torch.Tensor, N: int, beta: torch.Tensor, per_tensor: bool = False,
                     flags: int = 0, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. 7 + Eq. 11 on quantised activations.  fp32 [M,N], or int32 with FLAG_OUT_ACC_I32.
    `workspace` (workspace_bytes(OP_MATMUL, ...) bytes) is optional: see include/bitlinear.h."""
    M, K = codes.shape
    want_int = bool(flags & FLAG_OUT_ACC_I32)
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32 if want_int else torch.float32,
                          device=codes.device)
    _check(load_library().bitlinear_matmul(
        _ptr(codes, torch.int8), _ptr(gamma, torch.float32), _ptr(rowsum, torch.int32), M, K,
        _ptr(packed), N, _ptr(beta, torch.float32), _gran(per_tensor), flags, _ptr(out),
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()),
        "bitlinear_matmul")
    return out


def bitlinear_forward(X: torch.Tensor, packed: torch.Tensor, N: int, beta: torch.Tensor,
                      ln_eps: float = 1e-5, per_tensor: bool = False, flags: int = 0,
                      ln_gain=None, ln_bias=None, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. 11, the whole layer, from fp32 X [M,K] to fp32 Y [M,N]."""
    M, K = X.shape
    want_int = bool(flags & FLAG_OUT_ACC_I32)
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32 if want_int else torch.float32, device=X.device)
    ws = workspace if workspace is not None else _workspace(
        workspace_bytes(OP_FORWARD, M, N, K, per_tensor), X.device)
    _check(load_library().bitlinear_forward(
        _ptr(X, torch.float32), M, K, _ptr(packed), N, _ptr(beta, torch.float32),
        _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32), ln_eps, _gran(per_tensor),
        flags, _ptr(out), _ptr(ws), ws.numel(), _stream()), "bitlinear_forward")
    return out


def bitlinear_forward_static(X: torch.Tensor, packed: torch.Tensor, N: int, beta: torch.Tensor,
                             out: torch.Tensor, ln_eps: float = 1e-5, per_tensor: bool = False,
                             flags: int = 0, ln_gain=None, ln_bias=None) -> torch.Tensor:
    """bitlinear_forward with the library's own scratch array: nothing is allocated, here or in
    the library (the caller brings the output)."""
    M, K = X.shape
    _check(load_library().bitlinear_forward_static(
        _ptr(X, torch.float32), M, K, _ptr(packed), N, _ptr(beta, torch.float32),
        _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32), ln_eps, _gran(per_tensor),
        flags, _ptr(out), _stream()), "bitlinear_forward_static")
    return out


def probe_read(buf: torch.Tensor, workgroups: int = 256, threads: int = 448) -> None:
    """One launch that only reads `buf` (see bitlinear_probe_read): the floor a weight-streaming
    kernel is measured against."""
    _check(load_library().bitlinear_probe_read(_ptr(buf), buf.numel() * buf.element_size(), workgroups,
                                               threads, None, _stream()), "bitlinear_probe_read")


def bitlinear_backward_ste(dY: torch.Tensor, codes: torch.Tensor, gamma: torch.Tensor,
                           packed: torch.Tensor | None, beta: torch.Tensor, per_tensor: bool,
                           want_dx: bool = True, want_dw: bool = True,
                           workspace: torch.Tensor | None = None):
    """Section 2.2 (STE).  Returns (dX fp32 [M,K] or None, dW fp32 [N,K] or None)."""
    M, N = dY.shape
    K = codes.shape[1]
    dev = dY.device
    dX = torch.empty((M, K), dtype=torch.float32, device=dev) if want_dx else None
    dW = torch.empty((N, K), dtype=torch.float32, device=dev) if want_dw else None
    ws = workspace if workspace is not None else _workspace(
        workspace_bytes(OP_BACKWARD, M, N, K, per_tensor), dev)
    _check(load_library().bitlinear_backward_ste(
        _ptr(dY, torch.float32), M, N, K, _ptr(codes, torch.int8), _ptr(gamma, torch.float32),
        _gran(per_tensor), _ptr(packed), _ptr(beta, torch.float32), _ptr(dX), _ptr(dW), _ptr(ws),
        ws.numel(), _stream()), "bitlinear_backward_ste")
    return dX, dW


# ---- Group Quantization and Normalization (Eq. 13-15) ----------------------------------
def packed_bytes_grouped(N: int, K: int, groups_n: int, groups_k: int) -> int:
    return int(load_library().bitlinear_packed_bytes_grouped(N, K, groups_n, groups_k))


def workspace_bytes_grouped(op: int, M: int, N: int, K: int, groups_n: int, groups_k: int,
                            per_tensor: bool = False) -> int:
    return int(load_library().bitlinear_workspace_bytes_grouped(op, M, N, K, groups_n, groups_k,
                                                                _gran(per_tensor)))


def bitlinear_pack_weights_grouped(W: torch.Tensor, groups_n: int = 1, groups_k: int = 1,
                                   flags: int = 0):
    """Eq. 13.  Returns (packed blob, alpha [groups_n, groups_k], beta [groups_n, groups_k])."""
    N, K = W.shape
    nbytes = packed_bytes_grouped(N, K, groups_n, groups_k)
    packed = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=W.device)
    alpha = torch.empty((groups_n, groups_k), dtype=torch.float32, device=W.device)
    beta = torch.empty((groups_n, groups_k), dtype=torch.float32, device=W.device)
    ws = _workspace(workspace_bytes_grouped(OP_PACK, 0, N, K, groups_n, groups_k), W.device)
    _check(load_library().bitlinear_pack_weights_grouped(
        _ptr(W, torch.float32), N, K, groups_n, groups_k, flags, _ptr(packed), _ptr(alpha),
        _ptr(beta), _ptr(ws), ws.numel(), _stream()), "bitlinear_pack_weights_grouped")
    return packed, alpha, beta


def bitlinear_packed_to_canonical_grouped(packed: torch.Tensor, N: int, K: int,
                                          groups_k: int) -> torch.Tensor:
    out = torch.empty((N, K // 32), dtype=torch.int32, device=packed.device)
    _check(load_library().bitlinear_packed_to_canonical_grouped(
        _ptr(packed), N, K, groups_k, _ptr(out), _stream()), "bitlinear_packed_to_canonical_grouped")
    return out


def bitlinear_quant_act_grouped(X: torch.Tensor, groups_k: int, ln_eps: float = 1e-5,
                                per_tensor: bool = False, flags: int = 0, ln_gain=None,
                                ln_bias=None, want_xhat: bool = False):
    """Eq. 14-15.  Returns (codes [M,K], gamma [M,groups_k] or [groups_k], rowsum [M,groups_k],
    xhat or None)."""
    M, K = X.shape
    dev = X.device
    codes = torch.empty((M, K), dtype=torch.int8, device=dev)
    gamma = torch.empty((groups_k,) if per_tensor else (max(M, 1), groups_k), dtype=torch.float32,
                        device=dev)
    rowsum = torch.empty((max(M, 1), groups_k), dtype=torch.int32, device=dev)
    xhat = torch.empty((M, K), dtype=torch.float32, device=dev) if want_xhat else None
    ws = _workspace(workspace_bytes_grouped(OP_QUANT, M, 16, K, 1, groups_k, per_tensor), dev)
    _check(load_library().bitlinear_quant_act_grouped(
        _ptr(X, torch.float32), M, K, groups_k, _ptr(ln_gain, torch.float32),
        _ptr(ln_bias, torch.float32), ln_eps, _gran(per_tensor), flags, _ptr(codes), _ptr(gamma),
        _ptr(rowsum), _ptr(xhat), _ptr(ws), ws.numel(), _stream()), "bitlinear_quant_act_grouped")
    return codes, gamma, rowsum, xhat


def bitlinear_forward_grouped(X: torch.Tensor, packed: torch.Tensor, N: int, beta: torch.Tensor,
                              groups_n: int = 1, groups_k: int = 1, ln_eps: float = 1e-5,
                              per_tensor: bool = False, flags: int = 0, ln_gain=None, ln_bias=None,
                              out: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. 11 with the group parameters of Eq. 13-15."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    ws = _workspace(workspace_bytes_grouped(OP_FORWARD, M, N, K, groups_n, groups_k, per_tensor),
                    X.device)
    _check(load_library().bitlinear_forward_grouped(
        _ptr(X, torch.float32), M, K, _ptr(packed), N, groups_n, groups_k,
        _ptr(beta, torch.float32), _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32),
        ln_eps, _gran(per_tensor), flags, _ptr(out), _ptr(ws), ws.numel(), _stream()),
        "bitlinear_forward_grouped")
    return out


def bitlinear_layernorm_backward(dXhat: torch.Tensor, X: torch.Tensor, ln_eps: float = 1e-5,
                                 ln_gain=None, groups_k: int = 1, want_affine: bool = False,
                                 out: torch.Tensor | None = None):
    """Backward of Eq. 12 / Eq. 15.  Returns dX, or (dX, dgain, dbias) with want_affine."""
    M, K = X.shape
    dev = X.device
    dX = out if out is not None else torch.empty((M, K), dtype=torch.float32, device=dev)
    dgain = torch.empty(K, dtype=torch.float32, device=dev) if want_affine else None
    dbias = torch.empty(K, dtype=torch.float32, device=dev) if want_affine else None
    ws = _workspace(workspace_bytes_grouped(OP_LN_BACKWARD, M, 16, K, 1, groups_k), dev)
    _check(load_library().bitlinear_layernorm_backward(
        _ptr(dXhat, torch.float32), _ptr(X, torch.float32), M, K, groups_k,
        _ptr(ln_gain, torch.float32), ln_eps, _ptr(dX, torch.float32), _ptr(dgain), _ptr(dbias),
        _ptr(ws), ws.numel(), _stream()), "bitlinear_layernorm_backward")
    return (dX, dgain, dbias) if want_affine else dX


# ---- Eq. 6: the non-negative quantiser --------------------------------------------------
def bitlinear_weight_rowsums(packed: torch.Tensor, N: int, K: int) -> torch.Tensor:
    """wsum[n] = sum_k W~[n,k], int32 [N]."""
    out = torch.empty(N, dtype=torch.int32, device=packed.device)
    _check(load_library().bitlinear_weight_rowsums(_ptr(packed), N, K, _ptr(out), _stream()),
           "bitlinear_weight_rowsums")
    return out


def bitlinear_quant_act_nonneg(X: torch.Tensor, ln_eps: float = 1e-5, flags: int = 0, ln_gain=None,
                               ln_bias=None, want_xhat: bool = False, per_tensor: bool = False,
                               groups_k: int = 1):
    """Eq. 12 + Eq. 6 (per K-group: Eq. 14-15).  Returns (codes in 0..127, gamma, eta, rowsum, xhat or
    None); gamma and eta are [M, groups_k] per token, [groups_k] per tensor (flat for one group)."""
    M, K = X.shape
    dev = X.device
    codes = torch.empty((M, K), dtype=torch.int8, device=dev)
    n_par = groups_k if per_tensor else max(M, 1) * groups_k
    gamma = torch.empty(n_par, dtype=torch.float32, device=dev)
    eta = torch.empty(n_par, dtype=torch.float32, device=dev)
    rowsum = torch.empty(max(M, 1) * groups_k, dtype=torch.int32, device=dev)
    xhat = torch.empty((M, K), dtype=torch.float32, device=dev) if want_xhat else None
    ws = _workspace(workspace_bytes_grouped(OP_QUANT, M, 16, K, 1, groups_k, per_tensor), dev)
    lib = load_library()
    if groups_k == 1:
        _check(lib.bitlinear_quant_act_nonneg(
            _ptr(X, torch.float32), M, K, _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32),
            ln_eps, _gran(per_tensor), flags, _ptr(codes), _ptr(gamma), _ptr(eta), _ptr(rowsum),
            _ptr(xhat), _ptr(ws), ws.numel(), _stream()), "bitlinear_quant_act_nonneg")
    else:
        _check(lib.bitlinear_quant_act_grouped_nonneg(
            _ptr(X, torch.float32), M, K, groups_k, _ptr(ln_gain, torch.float32),
            _ptr(ln_bias, torch.float32), ln_eps, _gran(per_tensor), flags, _ptr(codes), _ptr(gamma),
            _ptr(eta), _ptr(rowsum), _ptr(xhat), _ptr(ws), ws.numel(), _stream()),
            "bitlinear_quant_act_grouped_nonneg")
    if groups_k > 1:
        shape = (groups_k,) if per_tensor else (max(M, 1), groups_k)
        gamma, eta, rowsum = gamma.view(shape), eta.view(shape), rowsum.view(max(M, 1), groups_k)
    return codes, gamma, eta, rowsum, xhat


def bitlinear_weight_rowsums_grouped(packed: torch.Tensor, N: int, K: int, groups_k: int) -> torch.Tensor:
    """wsum[g][n] = sum of W~[n, k] over the columns of K-group g, int32 [groups_k, N]."""
    out = torch.empty((groups_k, N), dtype=torch.int32, device=packed.device)
    _check(load_library().bitlinear_weight_rowsums_grouped(_ptr(packed), N, K, groups_k, _ptr(out),
                                                           _stream()), "bitlinear_weight_rowsums_grouped")
    return out


def bitlinear_matmul_nonneg(codes, gamma, eta, rowsum, packed, N: int, beta, wsum,
                            out: torch.Tensor | None = None, per_tensor: bool = False) -> torch.Tensor:
    M, K = codes.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=codes.device)
    _check(load_library().bitlinear_matmul_nonneg(
        _ptr(codes, torch.int8), _ptr(gamma, torch.float32), _ptr(eta, torch.float32),
        _ptr(rowsum, torch.int32), M, K, _ptr(packed), N, _ptr(beta, torch.float32),
        _ptr(wsum, torch.int32), _gran(per_tensor), 0, _ptr(out), _stream()),
        "bitlinear_matmul_nonneg")
    return out


def bitlinear_forward_nonneg(X: torch.Tensor, packed: torch.Tensor, N: int, beta: torch.Tensor,
                             wsum: torch.Tensor, ln_eps: float = 1e-5, flags: int = 0, ln_gain=None,
                             ln_bias=None, out: torch.Tensor | None = None, per_tensor: bool = False,
                             groups_n: int = 1, groups_k: int = 1) -> torch.Tensor:
    """Eq. 11 with the quantiser of Eq. 6 (with groups: Eq. 13-15, eta_g per K-group)."""
    M, K = X.shape
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    ws = _workspace(workspace_bytes_grouped(OP_FORWARD_NONNEG, M, N, K, groups_n, groups_k, per_tensor),
                    X.device)
    lib = load_library()
    if groups_n == 1 and groups_k == 1:
        _check(lib.bitlinear_forward_nonneg(
            _ptr(X, torch.float32), M, K, _ptr(packed), N, _ptr(beta, torch.float32),
            _ptr(wsum, torch.int32), _ptr(ln_gain, torch.float32), _ptr(ln_bias, torch.float32), ln_eps,
            _gran(per_tensor), flags, _ptr(out), _ptr(ws), ws.numel(), _stream()),
            "bitlinear_forward_nonneg")
    else:
        _check(lib.bitlinear_forward_grouped_nonneg(
            _ptr(X, torch.float32), M, K, _ptr(packed), N, groups_n, groups_k,
            _ptr(beta, torch.float32), _ptr(wsum, torch.int32), _ptr(ln_gain, torch.float32),
            _ptr(ln_bias, torch.float32), ln_eps, _gran(per_tensor), flags, _ptr(out), _ptr(ws),
            ws.numel(), _stream()), "bitlinear_forward_grouped_nonneg")
    return out


# ---- Mixtures of BitLinear layers ("experts") ------------------------------------------------
def _given(dev, t: torch.Tensor, dtype, *shape):
    """Pointer of an operand that has to lie on `dev`, be contiguous and have this type and shape.  (One test for all: a
    call of a few tokens is as long as what Python does for it.)"""
    if t.device == dev and t.shape == shape and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    if t.device != dev:
        raise BitLinearError(f"tensors on {dev} and {t.device}")
    if t.shape != shape:
        raise BitLinearError(f"expected a tensor of shape {shape}, got {tuple(t.shape)}")
    return _ptr(t, dtype)


def _here(t: torch.Tensor):
    """t's device, which has to be the current one: the launch goes to its current stream."""
    dev = t.device
    if dev.type != "cuda":
        raise BitLinearError("tensor is not on the GPU")
    if dev.index != torch._C._cuda_getDevice():
        raise BitLinearError(f"tensor on {dev}, current device {torch.cuda.current_device()}")
    return dev


def _queue(dev):
    """The current stream of the current device, which _here found to be `dev`."""
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _blob_bytes(N: int, K: int) -> int:
    """packed_bytes(N, K) of a shape that the call itself checks."""
    return (N + 15) // 16 * ((K + 511) // 512) * 1024


def workspace_bytes_experts(op: int, M: int, top_k: int, N: int, K: int, experts: int,
                            per_tensor: bool = False) -> int:
    return int(load_library().bitlinear_workspace_bytes_experts(op, M, top_k, N, K, experts, _gran(per_tensor)))


def _scratch(need: int, workspace: torch.Tensor | None, dev):
    """(pointer, bytes) of what the caller brought, or of a new buffer where one is needed."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = _workspace(need, dev)
    return _given(dev, workspace, torch.uint8, workspace.numel()), workspace.numel(), workspace


def bitlinear_pack_weights_experts(W: torch.Tensor, flags: int = 0):
    """Eq. 1-3, 12 for each expert of W [experts, N, K].  Returns (packed [experts, bytes], alpha [experts],
    beta [experts])."""
    lib, dev = load_library(), _here(W)
    E, N, K = W.shape
    nbytes = packed_bytes(N, K, flags)
    if nbytes == 0:
        _check(-2, "bitlinear_pack_weights")
    packed = torch.empty((E, nbytes), dtype=torch.uint8, device=dev)
    alpha = torch.empty(E, dtype=torch.float32, device=dev)
    beta = torch.empty(E, dtype=torch.float32, device=dev)
    ws = _workspace(workspace_bytes(OP_PACK, 0, N, K), dev)
    src = _ptr(W, torch.float32)
    for e in range(E):
        _check(lib.bitlinear_pack_weights(src + 4 * e * N * K, N, K, flags, packed.data_ptr() + e * nbytes,
                                          alpha.data_ptr() + 4 * e, beta.data_ptr() + 4 * e, _ptr(ws), ws.numel(),
                                          _queue(dev)), "bitlinear_pack_weights")
    return packed, alpha, beta


def bitlinear_route(expert: torch.Tensor, experts: int, workspace: torch.Tensor | None = None):
    """The router's choices int32 [M, top_k] sorted by expert.  Returns (order [M * top_k], position [M, top_k],
    offsets [experts + 1]), int32."""
    lib, dev = load_library(), _here(expert)
    M, top_k = expert.shape
    order = torch.empty(M * top_k, dtype=torch.int32, device=dev)
    position = torch.empty((M, top_k), dtype=torch.int32, device=dev)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=dev) if M else torch.zeros(
        experts + 1, dtype=torch.int32, device=dev)
    need = workspace_bytes_experts(OP_ROUTE, M, top_k, 0, 0, experts) if M * top_k > 4096 else 0
    ws, ws_bytes, _keep = _scratch(need, workspace, dev)
    _check(lib.bitlinear_route(_ptr(expert, torch.int32), M, top_k, experts, order.data_ptr(), position.data_ptr(),
                               offsets.data_ptr(), ws, ws_bytes, _queue(dev)), "bitlinear_route")
    return order, position, offsets


def _slots(codes, order, top_k):
    """(M, top_k, T): the slots that `codes` serve, through `order` or one a row."""
    M = codes.shape[0]
    if order is None:
        return M, 1, M
    return M, top_k, M * top_k


def bitlinear_matmul_experts(codes: torch.Tensor, gamma: torch.Tensor, rowsum: torch.Tensor, packed: torch.Tensor,
                             N: int, beta: torch.Tensor, offsets: torch.Tensor, order: torch.Tensor | None = None,
                             top_k: int = 1, per_tensor: bool = False, flags: int = 0,
                             out: torch.Tensor | None = None) -> torch.Tensor:
    """Eq. 7 + Eq. 11 with a weight matrix per expert: [slots, N] from the codes of tokens (through `order`, top_k slots
    a token) or of the slots themselves.  Slots without an expert are left as they were in `out`."""
    lib, dev = load_library(), _here(codes)
    M, top_k, T = _slots(codes, order, top_k)
    K, E = codes.shape[1], offsets.numel() - 1
    dtype = torch.int32 if flags & FLAG_OUT_ACC_I32 else torch.float32
    if out is None:
        out = torch.empty((T, N), dtype=dtype, device=dev)
    _check(lib.bitlinear_matmul_experts(
        _ptr(codes, torch.int8), _given(dev, gamma, torch.float32, 1 if per_tensor else M),
        _given(dev, rowsum, torch.int32, M), M, top_k, K, None if order is None else _given(dev, order, torch.int32, T),
        _given(dev, offsets, torch.int32, E + 1), E, _given(dev, packed, torch.uint8, E, _blob_bytes(N, K)), N,
        _given(dev, beta, torch.float32, E), _gran(per_tensor), flags, _given(dev, out, dtype, T, N), _queue(dev)),
        "bitlinear_matmul_experts")
    return out


def bitlinear_backward_ste_experts(dY: torch.Tensor, codes: torch.Tensor, gamma: torch.Tensor,
                                   packed: torch.Tensor | None, beta: torch.Tensor | None, offsets: torch.Tensor,
                                   order: torch.Tensor | None = None, top_k: int = 1, per_tensor: bool = False,
                                   want_dx: bool = True, want_dw: bool = True, workspace: torch.Tensor | None = None):
    """Section 2.2 (STE) for bitlinear_matmul_experts, dY bf16 [slots, N].  Returns (dX fp32 [slots, K] or None,
    dW fp32 [experts, N, K] or None)."""
    lib, dev = load_library(), _here(codes)
    M, top_k, T = _slots(codes, order, top_k)
    K, E, N = codes.shape[1], offsets.numel() - 1, dY.shape[1]
    dX = torch.empty((T, K), dtype=torch.float32, device=dev) if want_dx else None
    dW = (torch.empty if T else torch.zeros)((E, N, K), dtype=torch.float32, device=dev) if want_dw else None
    ws, ws_bytes, _keep = _scratch(workspace_bytes_experts(OP_BACKWARD, M, top_k, N, K, E, per_tensor), workspace, dev)
    _check(lib.bitlinear_backward_ste_experts(
        _given(dev, dY, torch.bfloat16, T, N), M, top_k, N, K, _ptr(codes, torch.int8),
        _given(dev, gamma, torch.float32, 1 if per_tensor else M), _gran(per_tensor),
        None if order is None else _given(dev, order, torch.int32, T), _given(dev, offsets, torch.int32, E + 1), E,
        None if packed is None else _given(dev, packed, torch.uint8, E, _blob_bytes(N, K)),
        None if beta is None else _given(dev, beta, torch.float32, E), _ptr(dX), _ptr(dW), ws, ws_bytes, _queue(dev)),
        "bitlinear_backward_ste_experts")
    return dX, dW


def bitlinear_combine(slots: torch.Tensor, position: torch.Tensor, weights: torch.Tensor | None = None,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """Slots [M * top_k, N] back to tokens [M, N], with the router's weights [M, top_k] (None: ones)."""
    lib, dev = load_library(), _here(slots)
    (M, top_k), N = position.shape, slots.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=dev)
    _check(lib.bitlinear_combine(
        _given(dev, slots, torch.float32, M * top_k, N), _given(dev, position, torch.int32, M, top_k),
        None if weights is None else _given(dev, weights, torch.float32, M, top_k), M, top_k, N,
        _given(dev, out, torch.float32, M, N), _queue(dev)), "bitlinear_combine")
    return out


def bitlinear_combine_backward(dY: torch.Tensor, slots: torch.Tensor | None, position: torch.Tensor,
                               weights: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """Gradient of bitlinear_combine.  Returns (dslots bf16 [M * top_k, N], dweights fp32 [M, top_k], or None without
    `slots`).  Rows of slots that no choice has are left as they were in `out`."""
    lib, dev = load_library(), _here(dY)
    (M, top_k), N = position.shape, dY.shape[1]
    if out is None:
        out = torch.empty((M * top_k, N), dtype=torch.bfloat16, device=dev)
    dweights = None if slots is None else torch.empty((M, top_k), dtype=torch.float32, device=dev)
    _check(lib.bitlinear_combine_backward(
        _given(dev, dY, torch.float32, M, N),
        None if slots is None else _given(dev, slots, torch.float32, M * top_k, N),
        _given(dev, position, torch.int32, M, top_k),
        None if weights is None else _given(dev, weights, torch.float32, M, top_k), M, top_k, N,
        _given(dev, out, torch.bfloat16, M * top_k, N), _ptr(dweights), _queue(dev)), "bitlinear_combine_backward")
    return out, dweights


def _function(fn: str) -> int:
    if fn not in FUNCTIONS:
        raise BitLinearError(f"unknown function {fn!r}: one of {', '.join(FUNCTIONS)}")
    return FUNCTIONS[fn]


def bitlinear_quant_nonlinear(U: torch.Tensor, fn: str = "gelu", ln_eps: float = 1e-5, per_tensor: bool = False,
                              checkpoint: bool = False, rows: torch.Tensor | None = None,
                              workspace: torch.Tensor | None = None):
    """Function, LayerNorm and quantiser of U [M, K] in one pass.  Returns (codes, gamma, rowsum, check int8 [M, K],
    check_scale fp32 [M, ceil(K / 128)]), the last two None without `checkpoint`.  rows: int32 [1], rows that exist.
    To train with a rectifier take "relu_marked" in both calls: the checkpoint of "relu" loses the gradient of every positive
    element that it rounds to zero."""
    lib, dev = load_library(), _here(U)
    M, K = U.shape
    codes = torch.empty((M, K), dtype=torch.int8, device=dev)
    gamma = torch.empty(1 if per_tensor else M, dtype=torch.float32, device=dev)
    if M == 0:
        gamma.fill_(1e-5)  # the call leaves it alone
    rowsum = torch.empty(M, dtype=torch.int32, device=dev)
    check = torch.empty((M, K), dtype=torch.int8, device=dev) if checkpoint else None
    scale = torch.empty((M, (K + 127) // 128), dtype=torch.float32, device=dev) if checkpoint else None
    need = workspace_bytes_experts(OP_QUANT_NONLINEAR, M, 1, 0, 0, 0, True) if per_tensor else 0
    ws, ws_bytes, _keep = _scratch(need, workspace, dev)
    _check(lib.bitlinear_quant_nonlinear(
        _ptr(U, torch.float32), M, K, _function(fn), ln_eps,
        None if rows is None else _given(dev, rows, torch.int32, 1), _gran(per_tensor), codes.data_ptr(),
        gamma.data_ptr(), rowsum.data_ptr(), _ptr(check), _ptr(scale), ws, ws_bytes, _queue(dev)),
        "bitlinear_quant_nonlinear")
    return codes, gamma, rowsum, check, scale


def bitlinear_nonlinear_backward(dXhat: torch.Tensor, check: torch.Tensor, check_scale: torch.Tensor, fn: str = "gelu",
                                 ln_eps: float = 1e-5, rows: torch.Tensor | None = None,
                                 dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """From the gradient of the normalised input of the next product to that of U, at the checkpoint: bf16 (as
    bitlinear_backward_ste_experts reads it) or fp32 (bitlinear_backward_ste)."""
    lib, dev = load_library(), _here(dXhat)
    M, K = dXhat.shape
    if dtype not in (torch.bfloat16, torch.float32):
        raise BitLinearError(f"expected torch.bfloat16 or torch.float32, got {dtype}")
    if out is None:
        out = torch.empty((M, K), dtype=dtype, device=dev)
    _check(lib.bitlinear_nonlinear_backward(
        _ptr(dXhat, torch.float32), _given(dev, check, torch.int8, M, K),
        _given(dev, check_scale, torch.float32, M, (K + 127) // 128), M, K, _function(fn), ln_eps,
        None if rows is None else _given(dev, rows, torch.int32, 1), BF16 if dtype == torch.bfloat16 else F32,
        _given(dev, out, dtype, M, K), _queue(dev)), "bitlinear_nonlinear_backward")
    return out
