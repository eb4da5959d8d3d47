"""ctypes binding: same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_HERE, "libaser.so")

EXPORTED_SYMBOLS = (
    "aser_pack_w4", "aser_repacked_bytes", "aser_repack_w4", "aser_unrepack_w4",
    "aser_quant_act", "aser_quant_act_bits", "aser_quant_act_ex", "aser_quant_act_ws",
    "aser_quant_workspace_bytes", "aser_quant_act_ws_launches", "aser_forward_act_launches", "aser_forward_host_parts", "aser_linear_kernel", "aser_linear_w4a8_lr_ld", "aser_forward_shared",
    "aser_linear_w4a8_lr_cat", "aser_forward_shared_cat_workspace_bytes", "aser_forward_shared_cat",
    "aser_forward_shared_workspace_bytes", "aser_construct", "aser_construct_workspace_bytes", "aser_linear_w4a8_lr", "aser_linear_w4a8", "aser_linear_w4a8_lr_simt", "aser_linear_w4a8_lr_static",
    "aser_workspace_bytes", "aser_workspace_init", "aser_check_status", "aser_forward",
    "aser_forward_host", "aser_linear_w4a8_lr_glu", "aser_forward_ffn_workspace_bytes", "aser_forward_ffn",
    "aser_adapters_plan_bytes", "aser_adapters_plan", "aser_quant_act_fine", "aser_adapters_add", "aser_adapters_workspace_bytes", "aser_forward_adapters", "aser_adapters_check_status",
    "aser_last_error", "aser_version",
)

if not os.path.exists(lib_path):
    raise ImportError(
        f"{lib_path} is missing: build it with `python -m paper_2411_07762_b200.build` "
        "(there is no fallback path)")
lib = C.CDLL(lib_path)

_P, _I, _Z = C.c_void_p, C.c_int, C.c_size_t
lib.aser_pack_w4.argtypes = [_P, _P, _I, _I, _P, _P, _P]
lib.aser_repacked_bytes.argtypes = [_I, _I]
lib.aser_repacked_bytes.restype = _Z
lib.aser_repack_w4.argtypes = [_P, _I, _I, _P, _P]
lib.aser_unrepack_w4.argtypes = [_P, _I, _I, _P, _P]
lib.aser_quant_act.argtypes = [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P]
lib.aser_quant_act_bits.argtypes = [_P, _P, _P, _I, _I, _I, _I, _P, _P, _P, _P]
lib.aser_quant_act_ex.argtypes = [_P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _P]
lib.aser_quant_workspace_bytes.argtypes = [_I, _I, _I]
lib.aser_quant_workspace_bytes.restype = _Z
lib.aser_forward_act_launches.argtypes = [_I, _I, _I]
lib.aser_forward_act_launches.restype = _I
lib.aser_forward_host_parts.argtypes = [_I, _I, _I, _P]
lib.aser_linear_kernel.argtypes = [_I, _I, _I]
lib.aser_quant_act_ws_launches.argtypes = [_I, _I]
lib.aser_quant_act_ws_launches.restype = _I
lib.aser_quant_act_ws.argtypes = [_P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _P, _Z, _P]
lib.aser_quant_act_fine.argtypes = [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _Z, _P]
lib.aser_linear_w4a8_lr_ld.argtypes = [_P, _P, _P, _P, _P, _I, _P, _I, _I, _I, _I, _P, _P, _P, _Z, _P]
lib.aser_forward_shared_workspace_bytes.argtypes = [_I, _P, _P, _I, _I]
lib.aser_forward_shared_workspace_bytes.restype = _Z
lib.aser_forward_shared.argtypes = [_P, _P, _P, _I, _P, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, _P, _Z, _P]
lib.aser_linear_w4a8_lr_cat.argtypes = [_P, _P, _P, _P, _P, _P, _I, _P, _I, _I, _I, _P, _P, _Z, _P]
lib.aser_forward_shared_cat_workspace_bytes.argtypes = [_I, _P, _I, _I, _I]
lib.aser_forward_shared_cat_workspace_bytes.restype = _Z
lib.aser_forward_shared_cat.argtypes = [_P, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _Z, _P]
lib.aser_linear_w4a8_lr.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P, _Z, _P]
lib.aser_linear_w4a8.argtypes = [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _Z, _P]
lib.aser_linear_w4a8_lr_simt.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P]
lib.aser_linear_w4a8_lr_static.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P]
lib.aser_workspace_bytes.argtypes = [_I, _I, _I, _I]
lib.aser_workspace_bytes.restype = _Z
lib.aser_workspace_init.argtypes = [_P, _Z, _P]
lib.aser_check_status.argtypes = [_P, _P]
lib.aser_forward.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P, _P, _P, _Z, _P]
lib.aser_forward_host.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                  _I, _I, _I, _I, _P, _Z, _P]
lib.aser_linear_w4a8_lr_glu.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _Z, _P]
lib.aser_forward_ffn_workspace_bytes.argtypes = [_I, _I, _I, _I, _I, _I]
lib.aser_forward_ffn_workspace_bytes.restype = _Z
lib.aser_forward_ffn.argtypes = [_P] * 11 + [_I] * 7 + [_P, _P, _Z, _P]
lib.aser_adapters_plan_bytes.argtypes = [_I, _I]
lib.aser_adapters_plan_bytes.restype = _Z
lib.aser_adapters_plan.argtypes = [_P, _I, _I, _P, _Z, _P]
lib.aser_adapters_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
lib.aser_adapters_workspace_bytes.restype = _Z
lib.aser_adapters_add.argtypes = [_P, _I, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _P, _I, _P, _I, _P, _Z, _P]
lib.aser_adapters_check_status.argtypes = [_P, _P]
lib.aser_forward_adapters.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P, _P, _P, _P, _P, _Z,
                                      _P, _P, _P, _P, _P, _Z, _I, _I, _P, _Z, _P]
lib.aser_construct_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
lib.aser_construct_workspace_bytes.restype = _Z
lib.aser_construct.argtypes = [_P, _P, _P, _I, _I, _I, _I, C.c_double, _I, _P, _P, _P, _P, _P, _P, _P, _I, _P, _Z, _P]
lib.aser_last_error.restype = C.c_char_p
lib.aser_version.restype = _I


class AserError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where} failed with code {code}: {last_error()}")


def last_error() -> str:
    return lib.aser_last_error().decode()


def version() -> int:
    return lib.aser_version()


# A pass of a few tokens is shorter on the GPU than its call from Python, so the call is kept lean: addresses
# and the stream go to ctypes as plain integers (a c_void_p object each and torch.cuda.current_stream()
# took 6 of the 15 us of a one-token pass).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _chk(rc: int, where: str):
    if rc != 0:
        raise AserError(rc, where)


def _dev(t: torch.Tensor, dtype, name: str):
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous CUDA tensor of {dtype}")
    return t


def pack_w4(W: torch.Tensor, s: torch.Tensor | None):
    """W fp16 [N,K], s fp32 [K] or None -> (Wq uint8 [N,K/2] canonical, w_scale fp32 [N])."""
    _dev(W, torch.float16, "W")
    N, K = W.shape
    Wq = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    w_scale = torch.empty((N,), dtype=torch.float32, device=W.device)
    _chk(lib.aser_pack_w4(_ptr(W), _ptr(s), N, K, _ptr(Wq), _ptr(w_scale), _stream()), "aser_pack_w4")
    return Wq, w_scale


def repacked_bytes(N: int, K: int) -> int:
    return int(lib.aser_repacked_bytes(N, K))


def repack_w4(Wq: torch.Tensor) -> torch.Tensor:
    _dev(Wq, torch.uint8, "Wq")
    N, K = Wq.shape[0], Wq.shape[1] * 2
    Wk = torch.empty((repacked_bytes(N, K),), dtype=torch.uint8, device=Wq.device)
    _chk(lib.aser_repack_w4(_ptr(Wq), N, K, _ptr(Wk), _stream()), "aser_repack_w4")
    return Wk


def unrepack_w4(Wk: torch.Tensor, N: int, K: int) -> torch.Tensor:
    _dev(Wk, torch.uint8, "Wk")
    Wq = torch.empty((N, K // 2), dtype=torch.uint8, device=Wk.device)
    _chk(lib.aser_unrepack_w4(_ptr(Wk), N, K, _ptr(Wq), _stream()), "aser_unrepack_w4")
    return Wq


def quant_act(X: torch.Tensor, s: torch.Tensor | None, L_A: torch.Tensor | None,
              out=None, act_bits: int = 8, t_pair: bool = False):
    """X fp16 [M,K] -> (Xq int8 [M,K], a_scale fp32 [M], T bf16 [M,r]).  act_bits != 8 goes
    through aser_quant_act_bits (codes of that width in the int8 container); t_pair through
    aser_quant_act_ex (T [M,2r]: a bf16 value and its bf16 remainder per entry)."""
    _dev(X, torch.float16, "X")
    M, K = X.shape
    r = 0 if L_A is None else L_A.shape[0]
    if out is None:
        Xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
        a_scale = torch.empty((M,), dtype=torch.float32, device=X.device)
        T = torch.empty((M, 2 * r if t_pair else r), dtype=torch.bfloat16, device=X.device)
    else:
        Xq, a_scale, T = out
    if t_pair:
        _chk(lib.aser_quant_act_ex(_ptr(X), _ptr(s), _ptr(L_A) if r else None, M, K, r, act_bits, 1,
                                   _ptr(Xq), _ptr(a_scale), _ptr(T) if r else None, _stream()),
             "aser_quant_act_ex")
        return Xq, a_scale, T
    if act_bits != 8:
        _chk(lib.aser_quant_act_bits(_ptr(X), _ptr(s), _ptr(L_A) if r else None, M, K, r, act_bits,
                                     _ptr(Xq), _ptr(a_scale), _ptr(T) if r else None, _stream()),
             "aser_quant_act_bits")
        return Xq, a_scale, T
    _chk(lib.aser_quant_act(_ptr(X), _ptr(s), _ptr(L_A) if r else None, M, K, r, _ptr(Xq),
                            _ptr(a_scale), _ptr(T) if r else None, _stream()), "aser_quant_act")
    return Xq, a_scale, T


def forward_act_launches(M: int, K: int, r: int) -> int:
    return int(lib.aser_forward_act_launches(M, K, r))


def quant_act_ws_launches(M: int, K: int) -> int:
    return int(lib.aser_quant_act_ws_launches(M, K))


def quant_workspace_bytes(M: int, K: int, r: int) -> int:
    return int(lib.aser_quant_workspace_bytes(M, K, r))


def quant_act_ws(X: torch.Tensor, s, L_A, ws: torch.Tensor | None = None, out=None,
                 act_bits: int = 8, t_pair: bool = False):
    """aser_quant_act_ws: quant_act with scratch memory (allocated here with torch when `ws` is
    None); L_A may be the stacked down projections of several layers, up to 512 rows."""
    _dev(X, torch.float16, "X")
    M, K = X.shape
    r = 0 if L_A is None else L_A.shape[0]
    if ws is None:
        ws = torch.empty((max(1024, quant_workspace_bytes(M, K, r)),), dtype=torch.uint8, device=X.device)
    if out is None:
        Xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
        a_scale = torch.empty((M,), dtype=torch.float32, device=X.device)
        T = torch.empty((M, 2 * r if t_pair else r), dtype=torch.bfloat16, device=X.device)
    else:
        Xq, a_scale, T = out
    _chk(lib.aser_quant_act_ws(_ptr(X), _ptr(s), _ptr(L_A) if r else None, M, K, r, act_bits,
                               1 if t_pair else 0, _ptr(Xq), _ptr(a_scale), _ptr(T) if r else None,
                               _ptr(ws), ws.numel(), _stream()), "aser_quant_act_ws")
    return Xq, a_scale, T


def quant_act_fine(X: torch.Tensor, s, L_A, ws: torch.Tensor | None = None, out=None):
    """aser_quant_act_fine: quant_act for what feeds another quantized layer (the quotients X / s enter T to 22 bits), the
    first step of a gated feed-forward block."""
    _dev(X, torch.float16, "X")
    M, K = X.shape
    r = 0 if L_A is None else L_A.shape[0]
    if ws is None:
        ws = torch.empty((max(1024, quant_workspace_bytes(M, K, r)),), dtype=torch.uint8, device=X.device)
    if out is None:
        Xq = torch.empty((M, K), dtype=torch.int8, device=X.device)
        a_scale = torch.empty((M,), dtype=torch.float32, device=X.device)
        T = torch.empty((M, r), dtype=torch.bfloat16, device=X.device)
    else:
        Xq, a_scale, T = out
    _chk(lib.aser_quant_act_fine(_ptr(X), _ptr(s), _ptr(L_A) if r else None, M, K, r, _ptr(Xq), _ptr(a_scale),
                                 _ptr(T) if r else None, _ptr(ws), ws.numel(), _stream()), "aser_quant_act_fine")
    return Xq, a_scale, T


def workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    return int(lib.aser_workspace_bytes(M, N, K, r))


def new_workspace(M: int, N: int, K: int, r: int, device="cuda") -> torch.Tensor:
    """Allocate (with torch) and zero a workspace for the given problem size."""
    nbytes = max(256, workspace_bytes(M, N, K, r))
    ws = torch.empty((nbytes,), dtype=torch.uint8, device=device)
    _chk(lib.aser_workspace_init(_ptr(ws), nbytes, _stream()), "aser_workspace_init")
    return ws


def check_status(ws: torch.Tensor) -> None:
    _chk(lib.aser_check_status(_ptr(ws), _stream()), "aser_check_status")


def linear_w4a8_lr(Xq, a_scale, Wk, w_scale, T, L_B, N: int, ws: torch.Tensor,
                   Y=None, acc_debug=None):
    M, K = Xq.shape
    r = 0 if L_B is None else L_B.shape[1]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    _chk(lib.aser_linear_w4a8_lr(_ptr(Xq), _ptr(a_scale), _ptr(Wk), _ptr(w_scale),
                                 _ptr(T) if r else None, _ptr(L_B) if r else None, M, N, K, r,
                                 _ptr(Y), _ptr(acc_debug), _ptr(ws), ws.numel(), _stream()),
         "aser_linear_w4a8_lr")
    return Y


def linear_w4a8_lr_ld(Xq, a_scale, Wk, w_scale, T_wide, col0: int, L_B, N: int, ws: torch.Tensor,
                      Y=None, acc_debug=None):
    """aser_linear_w4a8_lr_ld: the layer's T is columns [col0, col0 + r) of T_wide [M, R]."""
    M, K = Xq.shape
    r = L_B.shape[1]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    t_ptr = C.c_void_p(T_wide.data_ptr() + 2 * col0)
    _chk(lib.aser_linear_w4a8_lr_ld(_ptr(Xq), _ptr(a_scale), _ptr(Wk), _ptr(w_scale), t_ptr,
                                    T_wide.shape[1], _ptr(L_B), M, N, K, r, _ptr(Y), _ptr(acc_debug),
                                    _ptr(ws), ws.numel(), _stream()), "aser_linear_w4a8_lr_ld")
    return Y


def linear_w4a8(Xq, a_scale, Wk, w_scale, N: int, ws: torch.Tensor, Y=None, acc_debug=None):
    M, K = Xq.shape
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    _chk(lib.aser_linear_w4a8(_ptr(Xq), _ptr(a_scale), _ptr(Wk), _ptr(w_scale), M, N, K, _ptr(Y),
                              _ptr(acc_debug), _ptr(ws), ws.numel(), _stream()), "aser_linear_w4a8")
    return Y


ACTIVATIONS = {"silu": 0, "gelu_tanh": 1}


def _activation(name) -> int:
    if name not in ACTIVATIONS:
        raise ValueError("activation must be one of %s, not %r" % (", ".join(sorted(ACTIVATIONS)), name))
    return ACTIVATIONS[name]


def interleave_gate_up(gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
    """Rows of gate and up in turn: the order in which aser_linear_w4a8_lr_glu takes weights [F, K], scales [F] and up
    projections [F, r]."""
    if gate.shape != up.shape:
        raise ValueError("gate and up need the same shape")
    return torch.stack([gate, up], dim=1).reshape(2 * gate.shape[0], *gate.shape[1:]).contiguous()


def linear_w4a8_lr_glu(Xq, a_scale, Wk, w_scale, T, L_B, N: int, ws: torch.Tensor, activation: str = "silu", H=None):
    """aser_linear_w4a8_lr_glu: H fp16 [M, N / 2] = act(gate) * up of a projection whose N channels are gate and up in
    turn."""
    M, K = Xq.shape
    r = 0 if L_B is None else L_B.shape[1]
    if H is None:
        H = torch.empty((M, N // 2), dtype=torch.float16, device=Xq.device)
    elif _dev(H, torch.float16, "H").dim() != 2 or H.shape[0] < M or H.shape[1] != N // 2:
        raise ValueError("H needs %d rows of %d" % (M, N // 2))
    _chk(lib.aser_linear_w4a8_lr_glu(_ptr(Xq), _ptr(a_scale), _ptr(Wk), _ptr(w_scale), _ptr(T) if r else None,
                                     _ptr(L_B) if r else None, M, N, K, r, _activation(activation), _ptr(H), _ptr(ws),
                                     ws.numel(), _stream()), "aser_linear_w4a8_lr_glu")
    return H


def linear_w4a8_lr_simt(Xq, a_scale, Wq, w_scale, T, L_B, Y=None, acc_debug=None):
    M, K = Xq.shape
    N = Wq.shape[0]
    r = 0 if L_B is None else L_B.shape[1]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    _chk(lib.aser_linear_w4a8_lr_simt(_ptr(Xq), _ptr(a_scale), _ptr(Wq), _ptr(w_scale),
                                      _ptr(T) if r else None, _ptr(L_B) if r else None, M, N, K, r,
                                      _ptr(Y), _ptr(acc_debug), _stream()),
         "aser_linear_w4a8_lr_simt")
    return Y


def linear_w4a8_lr_static(Xq, a_scale, Wk, w_scale, T, L_B, N: int, Y=None, acc_debug=None):
    """aser_linear_w4a8_lr_static: same result as linear_w4a8_lr, no workspace argument (the
    library's built-in scratch array is used; at most 32 tokens per call)."""
    M, K = Xq.shape
    r = 0 if L_B is None else L_B.shape[1]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=Xq.device)
    _chk(lib.aser_linear_w4a8_lr_static(_ptr(Xq), _ptr(a_scale), _ptr(Wk), _ptr(w_scale),
                                        _ptr(T) if r else None, _ptr(L_B) if r else None, M, N, K,
                                        r, _ptr(Y), _ptr(acc_debug), _stream()),
         "aser_linear_w4a8_lr_static")
    return Y


def construct(W: torch.Tensor, s, X_cal: torch.Tensor, r: int, damping: float = 0.01, iterations: int = 0,
              want_S: bool = False, split_idx: torch.Tensor | None = None):
    """aser_construct: int4 weights and rank-r factors of one layer built on the device from W
    fp16 [N,K], s fp32 [K] and calibration tokens fp16 [n_cal,K].  Returns a dict with Wq, w_scale,
    L_A fp16 [r,K], L_B fp16 [N,r], sigma fp64 [r] and (want_S) the whitening factor S fp64 [K,K]."""
    _dev(W, torch.float16, "W")
    _dev(X_cal, torch.float16, "X_cal")
    N, K = W.shape
    n_cal = X_cal.shape[0]
    dev = W.device
    Wq = torch.empty((N, K // 2), dtype=torch.uint8, device=dev)
    w_scale = torch.empty((N,), dtype=torch.float32, device=dev)
    L_A = torch.empty((max(r, 1), K), dtype=torch.float16, device=dev)
    L_B = torch.empty((N, max(r, 1)), dtype=torch.float16, device=dev)
    sigma = torch.empty((max(r, 1),), dtype=torch.float64, device=dev)
    S = torch.empty((K, K), dtype=torch.float64, device=dev) if want_S else None
    n_split = 0 if split_idx is None else int(split_idx.numel())
    if n_split:
        _dev(split_idx, torch.int32, "split_idx")
    nbytes = int(lib.aser_construct_workspace_bytes(N, K, n_cal, r, n_split))
    ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=dev)
    _chk(lib.aser_construct(_ptr(W), _ptr(s), _ptr(X_cal), N, K, n_cal, r, float(damping), int(iterations),
                            _ptr(Wq), _ptr(w_scale), _ptr(L_A), _ptr(L_B), _ptr(sigma), _ptr(S),
                            _ptr(split_idx) if n_split else None, n_split, _ptr(ws),
                            ws.numel(), _stream()), "aser_construct")
    return dict(Wq=Wq, w_scale=w_scale, L_A=L_A[:r], L_B=L_B[:, :r].contiguous(), sigma=sigma[:r], S=S)


def pair_up_projection(L_B: torch.Tensor) -> torch.Tensor:
    """[L_B | L_B]: the up projection a linear kernel needs beside a T stored as bf16 pairs."""
    return torch.cat([L_B, L_B], dim=1).contiguous()


def pad_rank(L_A: torch.Tensor, L_B: torch.Tensor, multiple: int = 16):
    """Factors of a rank that is not a multiple of 16 (a per-layer rank chosen by the paper's
    singular-value threshold, Sec. 4.1) -> the same factors with zero rows appended to L_A
    [r,K] and zero columns to L_B [N,r], which adds exact zeros to T L_B^T.  The kernels take
    ranks in steps of 16 up to 256."""
    r = L_A.shape[0]
    if L_B.shape[1] != r:
        raise ValueError("L_A has %d rows but L_B has %d columns" % (r, L_B.shape[1]))
    rp = (r + multiple - 1) // multiple * multiple
    if rp == r:
        return L_A.contiguous(), L_B.contiguous()
    A = torch.zeros((rp, L_A.shape[1]), dtype=L_A.dtype, device=L_A.device)
    B = torch.zeros((L_B.shape[0], rp), dtype=L_B.dtype, device=L_B.device)
    A[:r] = L_A
    B[:, :r] = L_B
    return A, B


class AserLinear:
    """Device-resident operands of one ASER-quantized linear layer plus preallocated
    intermediates for up to `max_tokens` tokens.  __call__ runs aser_quant_act followed by
    aser_linear_w4a8_lr on the current stream."""

    def __init__(self, W: torch.Tensor, s: torch.Tensor | None, L_A: torch.Tensor | None,
                 L_B: torch.Tensor | None, max_tokens: int):
        self.N, self.K = W.shape
        self.r = 0 if L_A is None else L_A.shape[0]
        self.s, self.L_A, self.L_B = s, L_A, L_B
        self.Wq, self.w_scale = pack_w4(W, s)
        self.Wk = repack_w4(self.Wq)
        dev = W.device
        self.max_tokens = max_tokens
        self.Xq = torch.empty((max_tokens, self.K), dtype=torch.int8, device=dev)
        self.a_scale = torch.empty((max_tokens,), dtype=torch.float32, device=dev)
        self.T = torch.empty((max_tokens, max(self.r, 1)), dtype=torch.bfloat16, device=dev)
        self.Y = torch.empty((max_tokens, self.N), dtype=torch.float16, device=dev)
        self.X_dev = torch.empty((max_tokens, self.K), dtype=torch.float16, device=dev)
        self.ws = new_workspace(max_tokens, self.N, self.K, self.r, dev)

    def quant(self, X: torch.Tensor):
        """The activation step alone, with the kernels aser_forward runs at this shape."""
        M = X.shape[0]
        r = self.r
        if forward_act_launches(M, self.K, r or 16) == 1:       # (without a projection either step is one kernel: the same choice)
            _chk(lib.aser_quant_act(_ptr(X), _ptr(self.s), _ptr(self.L_A) if r else None, M, self.K, r,
                                    _ptr(self.Xq), _ptr(self.a_scale), _ptr(self.T) if r else None,
                                    _stream()), "aser_quant_act")
            return
        _chk(lib.aser_quant_act_ws(_ptr(X), _ptr(self.s), _ptr(self.L_A) if r else None, M, self.K, r,
                                   8, 0, _ptr(self.Xq), _ptr(self.a_scale), _ptr(self.T) if r else None,
                                   _ptr(self.ws), self.ws.numel(), _stream()), "aser_quant_act_ws")

    def linear(self, M: int, lowrank: bool = True, acc_debug=None):
        r = self.r if lowrank else 0
        if r:
            _chk(lib.aser_linear_w4a8_lr(_ptr(self.Xq), _ptr(self.a_scale), _ptr(self.Wk),
                                         _ptr(self.w_scale), _ptr(self.T), _ptr(self.L_B), M, self.N,
                                         self.K, r, _ptr(self.Y), _ptr(acc_debug), _ptr(self.ws),
                                         self.ws.numel(), _stream()), "aser_linear_w4a8_lr")
        else:
            _chk(lib.aser_linear_w4a8(_ptr(self.Xq), _ptr(self.a_scale), _ptr(self.Wk),
                                      _ptr(self.w_scale), M, self.N, self.K, _ptr(self.Y),
                                      _ptr(acc_debug), _ptr(self.ws), self.ws.numel(), _stream()),
                 "aser_linear_w4a8")

    def __call__(self, X: torch.Tensor, lowrank: bool = True, adapters: "AserAdapters | None" = None,
                 plan: "AdapterPlan | None" = None) -> torch.Tensor:
        """One forward pass through aser_forward (quantization and linear kernel overlapped); with `adapters` and the
        `plan` of the batch through aser_forward_adapters (X may then not be the layer's own output, which is written before
        the adapters read X)."""
        M = X.shape[0]
        if adapters is not None:
            return adapters._forward(self, X, plan, lowrank)
        if plan is not None:
            raise ValueError("a plan without adapters")
        assert M <= self.max_tokens
        r = self.r if lowrank else 0       # the plain W4A8 control: the same entry point at rank 0
        s, Y, ws = self.s, self.Y, self.ws
        rc = lib.aser_forward(X.data_ptr(), None if s is None else s.data_ptr(), self.L_A.data_ptr() if r else None,
                              self.Wk.data_ptr(), self.w_scale.data_ptr(), self.L_B.data_ptr() if r else None,
                              M, self.N, self.K, r, self.Xq.data_ptr(), self.a_scale.data_ptr(),
                              self.T.data_ptr() if r else None, Y.data_ptr(), ws.data_ptr(), ws.numel(), _stream())
        if rc != 0:
            raise AserError(rc, "aser_forward")
        return Y[:M]                       # (a slice: narrow costs a microsecond more)

    def forward_host(self, X_host: torch.Tensor, Y_host: torch.Tensor):
        """Host fp16 X [M,K] (pinned) -> host fp16 Y [M,N] through aser_forward_host."""
        forward_host(self, X_host, Y_host)


class AserSharedInput:
    """Layers that read the same activation and share the smoothing vector (query/key/value, or
    gate/up): one activation pass for all of them through aser_forward_shared.  Built from
    AserLinear objects; their packed weights and factors are used in place."""

    def __init__(self, layers, max_tokens: int):
        self.layers = list(layers)
        first = self.layers[0]
        self.K, self.s = first.K, first.s
        for L in self.layers:
            if L.K != self.K or (L.s is not first.s and not torch.equal(L.s, first.s)):
                raise ValueError("layers of a shared-input group need the same K and smoothing vector")
        dev = first.Wk.device
        self.n = len(self.layers)
        self.r = [L.r for L in self.layers]
        self.N = [L.N for L in self.layers]
        self.r_total = sum(self.r)
        self.L_A = torch.cat([L.L_A for L in self.layers if L.r], dim=0).contiguous() if self.r_total else None
        self.max_tokens = max_tokens
        self.Xq = torch.empty((max_tokens, self.K), dtype=torch.int8, device=dev)
        self.a_scale = torch.empty((max_tokens,), dtype=torch.float32, device=dev)
        self.T = torch.empty((max_tokens, max(self.r_total, 1)), dtype=torch.bfloat16, device=dev)
        self.Y = [torch.empty((max_tokens, n), dtype=torch.float16, device=dev) for n in self.N]
        arr_i = C.c_int * self.n
        arr_p = C.c_void_p * self.n
        self._N, self._r = arr_i(*self.N), arr_i(*self.r)
        self._Wk = arr_p(*[L.Wk.data_ptr() for L in self.layers])
        self._ws = arr_p(*[L.w_scale.data_ptr() for L in self.layers])
        self._LB = arr_p(*[(L.L_B.data_ptr() if L.r else None) for L in self.layers])
        self._Y = arr_p(*[y.data_ptr() for y in self.Y])
        nbytes = int(lib.aser_forward_shared_workspace_bytes(self.n, self._N, self._r, max_tokens, self.K))
        if nbytes == 0:
            raise ValueError("unsupported shapes for a shared-input group")
        self.ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)
        _chk(lib.aser_workspace_init(_ptr(self.ws), nbytes, _stream()), "aser_workspace_init")

    def quant(self, X: torch.Tensor):
        """The activation pass of the group alone (aser_quant_act_ws with the stacked L_A)."""
        M = X.shape[0]
        if forward_act_launches(M, self.K, self.r_total or 16) == 1 and self.r_total <= 256:
            _chk(lib.aser_quant_act(_ptr(X), _ptr(self.s), _ptr(self.L_A), M, self.K, self.r_total,
                                    _ptr(self.Xq), _ptr(self.a_scale), _ptr(self.T) if self.r_total else None,
                                    _stream()), "aser_quant_act")
            return
        _chk(lib.aser_quant_act_ws(_ptr(X), _ptr(self.s), _ptr(self.L_A), M, self.K, self.r_total, 8, 0,
                                   _ptr(self.Xq), _ptr(self.a_scale), _ptr(self.T) if self.r_total else None,
                                   _ptr(self.ws), self.ws.numel(), _stream()), "aser_quant_act_ws")

    def __call__(self, X: torch.Tensor):
        """Returns the layers' outputs [M, N_l] (views of preallocated buffers)."""
        M = X.shape[0]
        assert M <= self.max_tokens
        _chk(lib.aser_forward_shared(_ptr(X), _ptr(self.s), _ptr(self.L_A), self.n, self._Wk, self._ws,
                                     self._LB, self._N, self._r, M, self.K, _ptr(self.Xq),
                                     _ptr(self.a_scale), _ptr(self.T) if self.r_total else None, self._Y,
                                     _ptr(self.ws), self.ws.numel(), _stream()), "aser_forward_shared")
        return [y[:M] for y in self.Y]



class AserSharedInputCat(AserSharedInput):
    """A shared-input group stored as one fused projection: the layers' packed weights, scales and
    up projections are concatenated along N (copies are made here) and the outputs are column
    ranges of one [M, sum N] buffer, so that a single linear launch serves the group
    (aser_forward_shared_cat).  Needs every N a multiple of 128 and one rank for all layers."""

    def __init__(self, layers, max_tokens: int):
        super().__init__(layers, max_tokens)
        if len(set(self.r)) != 1 or any(n % 128 for n in self.N) or self.n > 4:
            raise ValueError("a concatenated group needs one rank, N multiples of 128 and at most four layers")
        dev = self.layers[0].Wk.device
        self.r1 = self.r[0]
        self.N_total = sum(self.N)
        self.Wk_cat = torch.cat([L.Wk.reshape(-1) for L in self.layers]).contiguous()
        self.w_scale_cat = torch.cat([L.w_scale for L in self.layers]).contiguous()
        self.L_B_cat = torch.cat([L.L_B for L in self.layers], dim=0).contiguous() if self.r1 else None
        self.Y_cat = torch.empty((max_tokens, self.N_total), dtype=torch.float16, device=dev)
        nbytes = int(lib.aser_forward_shared_cat_workspace_bytes(self.n, self._N, self.r1, max_tokens, self.K))
        if nbytes == 0:
            raise ValueError("unsupported shapes for a concatenated shared-input group")
        if nbytes > self.ws.numel():
            self.ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)
            _chk(lib.aser_workspace_init(_ptr(self.ws), nbytes, _stream()), "aser_workspace_init")

    def _views(self, M: int):
        out, col = [], 0
        for n in self.N:
            out.append((self.Y_cat if M == self.max_tokens else self.Y_cat[:M]).narrow(1, col, n))
            col += n
        return out

    def linear(self, M: int):
        """The linear step alone on the codes and T of the last activation pass."""
        _chk(lib.aser_linear_w4a8_lr_cat(_ptr(self.Xq), _ptr(self.a_scale), _ptr(self.Wk_cat),
                                         _ptr(self.w_scale_cat), _ptr(self.T) if self.r1 else None,
                                         _ptr(self.L_B_cat) if self.r1 else None, self.n, self._N, self.r1,
                                         M, self.K, _ptr(self.Y_cat), _ptr(self.ws), self.ws.numel(),
                                         _stream()), "aser_linear_w4a8_lr_cat")
        return self._views(M)

    def __call__(self, X: torch.Tensor):
        """Returns the layers' outputs as column ranges of the fused output [M, sum N]."""
        M = X.shape[0]
        assert M == self.max_tokens, "the fused output buffer is laid out for max_tokens rows"
        _chk(lib.aser_forward_shared_cat(_ptr(X), _ptr(self.s), _ptr(self.L_A), self.n, _ptr(self.Wk_cat),
                                         _ptr(self.w_scale_cat), _ptr(self.L_B_cat) if self.r1 else None,
                                         self._N, self.r1, M, self.K, _ptr(self.Xq), _ptr(self.a_scale),
                                         _ptr(self.T) if self.r_total else None, _ptr(self.Y_cat),
                                         _ptr(self.ws), self.ws.numel(), _stream()), "aser_forward_shared_cat")
        return self._views(M)


def _rows(v: torch.Tensor, shape: tuple, name: str, device: int) -> int:
    """Elements between the rows of an fp16 matrix of that shape on that GPU whose rows are contiguous."""
    if v.shape != shape or v.dtype is not torch.float16 or v.get_device() != device:
        raise TypeError("%s: need a tensor of torch.float16, [%d, %d], on the current GPU" % (name, *shape))
    ld, step = v.stride()
    if shape[0] <= 1 and (step == 1 or shape[1] <= 1):
        return shape[1]                                 # (the stride of a dimension of one element says nothing)
    if step == 1 and ld >= shape[1]:
        return ld
    raise TypeError("%s: rows need to be contiguous and apart" % name)


class AdapterPlan:
    """The tokens of a batch by adapter (aser_adapters_plan): made once, used by the adapters of every layer of a step.
    `update` follows new slots in the same memory, also inside a captured graph."""

    def __init__(self, slot: torch.Tensor, n_slots: int):
        self.M, self.n_slots = slot.numel(), n_slots
        nbytes = int(lib.aser_adapters_plan_bytes(self.M, n_slots))
        if nbytes == 0:
            raise ValueError("unsupported number of tokens or adapters")
        self.nbytes = nbytes
        self.device = slot.get_device()
        self.data = torch.empty((nbytes,), dtype=torch.uint8, device=slot.device)
        self.update(slot)

    def update(self, slot: torch.Tensor) -> "AdapterPlan":
        _dev(slot, torch.int32, "slot")
        if slot.dim() != 1 or slot.numel() != self.M:
            raise ValueError("slot needs one dimension of %d tokens" % self.M)
        if slot.get_device() != self.device or self.device != torch._C._cuda_getDevice():
            raise ValueError("slot and plan need to be on the current GPU")
        _chk(lib.aser_adapters_plan(_ptr(slot), self.M, self.n_slots, _ptr(self.data), self.nbytes, _stream()),
             "aser_adapters_plan")
        return self

    def check_status(self) -> None:
        """Raises if a bounded wait of an adapter call with this plan gave up (aser_adapters_check_status; synchronises)."""
        if self.M:
            _chk(lib.aser_adapters_check_status(_ptr(self.data), _stream()), "aser_adapters_check_status")


class AserAdapters:
    """A pool of low-rank adapters of one projection: A fp16 [slots, r, K], B fp16 [slots, N, r], with a rank each (int32
    [slots], multiples of 16; None: all r) and a factor each (fp32 [slots]; None: ones).  The pool's tensors are used in place,
    so an adapter is exchanged by writing to them."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None,
                 ranks: torch.Tensor | None = None):
        _dev(A, torch.float16, "A")
        _dev(B, torch.float16, "B")
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
            raise ValueError("need A [slots, r, K] and B [slots, N, r]")
        self.n_slots, self.r, self.K = A.shape
        self.N = B.shape[1]
        for v, dtype, name in ((scale, torch.float32, "scale"), (ranks, torch.int32, "ranks")):
            if v is not None and _dev(v, dtype, name).shape != (self.n_slots,):
                raise ValueError("%s needs one element per adapter" % name)
        self.A, self.B, self.scale, self.ranks = A, B, scale, ranks
        self.device = A.get_device()
        if any(v is not None and v.get_device() != self.device for v in (B, scale, ranks)):
            raise ValueError("a pool's tensors need to be on one GPU")
        self._ws_bytes = {}

    def plan(self, slot: torch.Tensor) -> AdapterPlan:
        """slot int32 [M]: the adapter of each token, anything outside 0 .. slots - 1 for none."""
        return AdapterPlan(slot, self.n_slots)

    def _check_plan(self, plan, M: int, device: int):
        if plan is None or plan.M != M or plan.n_slots != self.n_slots:
            raise ValueError("need a plan of %d tokens and %d adapters" % (M, self.n_slots))
        if not plan.device == self.device == device:
            raise ValueError("adapters and plan need to be on the current GPU")

    def _workspace(self, M: int):
        """What a call of many tokens keeps between its two launches: torch's memory of the current stream."""
        nbytes = self._ws_bytes.get(M)
        if nbytes is None:
            nbytes = self._ws_bytes[M] = lib.aser_adapters_workspace_bytes(M, self.N, self.K, self.r, self.n_slots)
        return None if nbytes == 0 else torch.empty((nbytes,), dtype=torch.uint8, device=self.A.device)

    def add(self, X: torch.Tensor, Y: torch.Tensor, plan: AdapterPlan, out: torch.Tensor | None = None) -> torch.Tensor:
        """out = Y + scale B (A x) by each token's adapter; X fp16 [M, K], Y and out fp16 [M, N], rows of which may be apart
        (a column range of a fused projection).  Without `out` in place; what is written may not overlap X."""
        # (a call of a few tokens is shorter on the GPU than from here, as everywhere in this file)
        M, device = X.shape[0], torch._C._cuda_getDevice()
        ldx = _rows(X, (M, self.K), "X", device)
        ldy = _rows(Y, (M, self.N), "Y", device)
        y_at = Y.data_ptr()
        if out is None:
            out, ldo, out_at = Y, ldy, y_at
        else:
            ldo, out_at = _rows(out, (M, self.N), "out", device), out.data_ptr()
        self._check_plan(plan, M, device)
        scale, ranks = self.scale, self.ranks
        ws = self._workspace(M) if M > 32 else None
        rc = lib.aser_adapters_add(X.data_ptr(), ldx, self.A.data_ptr(), self.B.data_ptr(),
                                   None if ranks is None else ranks.data_ptr(), None if scale is None else scale.data_ptr(),
                                   plan.data.data_ptr(), plan.nbytes, M, self.N, self.K, self.r, self.n_slots, y_at, ldy, out_at,
                                   ldo, None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream())
        if rc != 0:
            raise AserError(rc, "aser_adapters_add")
        return out

    def _forward(self, layer: "AserLinear", X: torch.Tensor, plan: AdapterPlan, lowrank: bool) -> torch.Tensor:
        M = X.shape[0]
        if M > layer.max_tokens or (layer.K, layer.N) != (self.K, self.N):
            raise ValueError("%d tokens of a [%d, %d] layer and adapters of [%d, %d]: they do not fit"
                             % (M, layer.N, layer.K, self.N, self.K))
        device = torch._C._cuda_getDevice()
        if _rows(X, (M, self.K), "X", device) != self.K:
            raise TypeError("X: rows need to be adjacent")
        self._check_plan(plan, M, device)
        if layer.Wk.get_device() != device:
            raise ValueError("the layer needs to be on the current GPU")
        r = layer.r if lowrank else 0
        ws = self._workspace(M)
        rc = lib.aser_forward_adapters(X.data_ptr(), _ptr(layer.s), layer.L_A.data_ptr() if r else None, layer.Wk.data_ptr(),
                                       layer.w_scale.data_ptr(), layer.L_B.data_ptr() if r else None, M, self.N, self.K, r,
                                       layer.Xq.data_ptr(), layer.a_scale.data_ptr(), layer.T.data_ptr() if r else None,
                                       layer.Y.data_ptr(), layer.ws.data_ptr(), layer.ws.numel(), self.A.data_ptr(),
                                       self.B.data_ptr(), _ptr(self.ranks), _ptr(self.scale), plan.data.data_ptr(), plan.nbytes,
                                       self.r, self.n_slots, _ptr(ws), 0 if ws is None else ws.numel(), _stream())
        if rc != 0:
            raise AserError(rc, "aser_forward_adapters")
        return layer.Y[:M]


def _on_current_gpu(**tensors):
    """Tensors that a kernel launched now would read lie on the GPU that it would run on."""
    device = torch._C._cuda_getDevice()
    for name, v in tensors.items():
        if v is not None and v.get_device() != device:
            raise ValueError("%s needs to be on the current GPU" % name)


class AserGatedFFN:
    """Gated feed-forward block of three ASER-quantized layers, Y = down(act(gate(X)) * up(X)), through
    aser_forward_ffn; device-resident operands and a workspace for up to `max_tokens` tokens.

    W_gate, W_up fp16 [F,K] with one smoothing vector s [K] (or None) and one pair of factors for both: L_A [r,K], L_B [2F,r]
    whose first F rows are gate's (None for no low-rank term); W_down fp16 [N,F] with s_down [F], L_A_down [r',F],
    L_B_down [N,r'].  The packed gate and up channels are stored in turn.  A block has one workspace and one output buffer: calls that
    overlap in time, and graphs that may run at the same time, need a block each."""

    def __init__(self, W_gate, W_up, s, L_A, L_B, W_down, s_down, L_A_down, L_B_down, max_tokens: int,
                 activation: str = "silu"):
        _on_current_gpu(W_gate=W_gate, W_up=W_up, s=s, L_A=L_A, L_B=L_B, W_down=W_down, s_down=s_down, L_A_down=L_A_down,
                        L_B_down=L_B_down)
        self.F, self.K = W_gate.shape
        self.N = W_down.shape[0]
        if W_up.shape != W_gate.shape or W_down.shape[1] != self.F:
            raise ValueError("gate and up need the same shape, and down as many columns as they have rows")
        if (L_A is None) != (L_B is None) or (L_A_down is None) != (L_B_down is None):
            raise ValueError("L_A and L_B come together")
        self.activation = _activation(activation)
        self.max_tokens = max_tokens
        self.r = 0 if L_A is None else L_A.shape[0]
        self.r_down = 0 if L_A_down is None else L_A_down.shape[0]
        for A, B, k, n, r, what in ((L_A, L_B, self.K, 2 * self.F, self.r, "gate and up"),
                                    (L_A_down, L_B_down, self.F, self.N, self.r_down, "down")):
            if r and (tuple(A.shape) != (r, k) or tuple(B.shape) != (n, r)):
                raise ValueError("factors of %s: need L_A [%d, %d] and L_B [%d, %d]" % (what, r, k, n, r))
        for v, k, name in ((s, self.K, "s"), (s_down, self.F, "s_down")):
            if v is not None and (_dev(v, torch.float32, name).shape != (k,)):
                raise ValueError("%s needs %d elements" % (name, k))
        nbytes = int(lib.aser_forward_ffn_workspace_bytes(max_tokens, self.K, self.F, self.N, self.r, self.r_down))
        if nbytes == 0:
            raise ValueError("unsupported shapes for a feed-forward block")
        dev = W_gate.device
        self.s, self.s_down = s, s_down
        Wq, self.w_scale = pack_w4(interleave_gate_up(W_gate, W_up), s)         # (the canonical form is not kept: no call reads it)
        self.Wk = repack_w4(Wq)
        self.L_A = None if L_A is None else _dev(L_A, torch.float16, "L_A")
        self.L_B = None if L_B is None else interleave_gate_up(*_dev(L_B, torch.float16, "L_B").chunk(2))
        Wq, self.w_scale_down = pack_w4(_dev(W_down, torch.float16, "W_down"), s_down)
        self.Wk_down = repack_w4(Wq)
        self.L_A_down = None if L_A_down is None else _dev(L_A_down, torch.float16, "L_A_down")
        self.L_B_down = None if L_B_down is None else _dev(L_B_down, torch.float16, "L_B_down")
        self.Y = torch.empty((max_tokens, self.N), dtype=torch.float16, device=dev)
        self.ws = torch.empty((nbytes,), dtype=torch.uint8, device=dev)
        _chk(lib.aser_workspace_init(_ptr(self.ws), nbytes, _stream()), "aser_workspace_init")

    def __call__(self, X: torch.Tensor) -> torch.Tensor:
        """Y [M, N] (a view of a preallocated buffer) of X fp16 [M, K], M up to max_tokens."""
        device = torch._C._cuda_getDevice()
        if X.dtype != torch.float16 or X.get_device() != device or not X.is_contiguous() or X.dim() != 2 or X.shape[1] != self.K:
            raise TypeError("X: need a contiguous tensor of torch.float16, [M, %d], on the current GPU" % self.K)
        if self.Y.get_device() != device:
            raise ValueError("the block needs to be on the current GPU")
        M = X.shape[0]
        if M > self.max_tokens:
            raise ValueError("%d tokens, but the block was made for %d" % (M, self.max_tokens))
        rc = lib.aser_forward_ffn(X.data_ptr(), _ptr(self.s), _ptr(self.L_A), self.Wk.data_ptr(), self.w_scale.data_ptr(),
                                  _ptr(self.L_B), _ptr(self.s_down), _ptr(self.L_A_down), self.Wk_down.data_ptr(),
                                  self.w_scale_down.data_ptr(), _ptr(self.L_B_down), M, self.K, self.F, self.N, self.r,
                                  self.r_down, self.activation, self.Y.data_ptr(), self.ws.data_ptr(), self.ws.numel(),
                                  _stream())
        if rc != 0:
            raise AserError(rc, "aser_forward_ffn")
        return self.Y[:M]


def forward_host(layer: AserLinear, X_host: torch.Tensor, Y_host: torch.Tensor):
    M = X_host.shape[0]
    r = layer.r
    _chk(lib.aser_forward_host(_ptr(X_host), _ptr(Y_host), _ptr(layer.X_dev), _ptr(layer.Xq),
                               _ptr(layer.a_scale), _ptr(layer.T), _ptr(layer.Y), _ptr(layer.s),
                               _ptr(layer.L_A) if r else None, _ptr(layer.Wk), _ptr(layer.w_scale),
                               _ptr(layer.L_B) if r else None, M, layer.N, layer.K, r,
                               _ptr(layer.ws), layer.ws.numel(), _stream()), "aser_forward_host")
