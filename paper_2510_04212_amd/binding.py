"""Thin ctypes binding over the C ABI declared in include/attn.h.

Argument marshalling only: every step of the attention forward/backward runs in the HIP
kernels of libattn_gfx950.so.  torch is used for device memory and for the current stream.
There is no fallback: if the library has not been built, importing this module raises.
"""
import ctypes
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn_gfx950.so")

STANDARD = 0
MITIGATED = 1
MITIGATED_ROW = 2
DEFAULT_BETA = 2.0
DEFAULT_EPS = 1e-3

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it first with `python -m paper_2510_04212_amd.build` "
        "(there is no CPU or PyTorch fallback for the attention kernels)")

_lib = ctypes.CDLL(LIB_PATH)

_vp, _i, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_lib.attn_fwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_fwd.restype = _i
_lib.attn_fwd_ex.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _f, _i, _f, _f, _vp]
_lib.attn_fwd_ex.restype = _i
_lib.attn_fwd_opt.argtypes = [_vp] * 8 + [_i, _i, _i, _i, _i, _f, _i, _f, _f, ctypes.c_uint, _vp]
_lib.attn_fwd_opt.restype = _i
_lib.attn_delta.argtypes = [_vp, _vp, _vp, _i, _i, _i, _i, _vp]
_lib.attn_delta.restype = _i
_lib.attn_delta_hp.argtypes = [_vp, _vp, _vp, _i, _i, _i, _i, _vp]
_lib.attn_delta_hp.restype = _i
_lib.attn_delta_recompute.argtypes = [_vp] * 6 + [_i, _i, _i, _i, _i, _f, _vp]
_lib.attn_delta_recompute.restype = _i
_ll = ctypes.c_longlong
_lib.attn_fwd_strided.argtypes = [_vp] * 5 + [_ll, _ll, _ll, _i, _i, _i, _i, _i, _f, _i, _f, _f, _vp]
_lib.attn_fwd_strided.restype = _i
_lib.attn_bwd_strided.argtypes = [_vp] * 9 + [_vp, _sz, _ll, _ll, _ll, _i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_bwd_strided.restype = _i
_lib.attn_fwd_gqa.argtypes = [_vp] * 5 + [_i, _i, _i, _i, _i, _i, _f, _i, _f, _f, _vp]
_lib.attn_fwd_gqa.restype = _i
_lib.attn_bwd_gqa.argtypes = [_vp] * 9 + [_vp, _sz, _i, _i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_bwd_gqa.restype = _i
_lib.attn_fwd_rect.argtypes = [_vp] * 5 + [_i, _i, _i, _i, _i, _i, _f, _i, _f, _f, _vp]
_lib.attn_fwd_rect.restype = _i
_lib.attn_bwd_rect.argtypes = [_vp] * 9 + [_vp, _sz, _i, _i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_bwd_rect.restype = _i
_lib.attn_fwd_ws.argtypes = [_vp] * 6 + [_sz, _ll, _ll, _ll] + [_i] * 7 + [_f, _i, _f, _f, _vp]
_lib.attn_fwd_ws.restype = _i
_lib.attn_fwd_workspace_bytes.argtypes = [_i] * 7
_lib.attn_fwd_workspace_bytes.restype = _sz
_lib.attn_bwd.argtypes = [_vp] * 9 + [_vp, _sz, _i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_bwd.restype = _i
_lib.attn_bwd_noalloc.argtypes = [_vp] * 9 + [_i, _i, _i, _i, _i, _f, _i, _vp]
_lib.attn_bwd_noalloc.restype = _i
_lib.attn_bwd_noalloc_max_rows.argtypes = []
_lib.attn_bwd_noalloc_max_rows.restype = _sz
_lib.attn_bwd_dkdv.argtypes = [_vp] * 8 + [_i, _i, _i, _i, _i, _f, _vp]
_lib.attn_bwd_dkdv.restype = _i
_lib.attn_bwd_dq.argtypes = [_vp] * 7 + [_i, _i, _i, _i, _i, _f, _vp]
_lib.attn_bwd_dq_delta.argtypes = [_vp] * 8 + [_i, _i, _i, _i, _i, _f, _vp]
_lib.attn_bwd_dq_delta.restype = _i
_lib.attn_bwd_dq.restype = _i
_lib.attn_bwd_workspace_bytes.argtypes = [_i, _i, _i, _i]
_lib.attn_bwd_workspace_bytes.restype = _sz
_lib.attn_rope.argtypes = [_vp] * 6 + [_ll, _vp] + [_i] * 7 + [_f, _i, _vp]
_lib.attn_rope.restype = _i
_d = ctypes.c_double
_lib.attn_rope_frequencies.argtypes = [_vp, _vp, _i, _d, _i, _d, _d, _d, _d]
_lib.attn_rope_frequencies.restype = _i
_lib.attn_cache_append.argtypes = [_vp] * 9 + [_i] * 5 + [_vp]
_lib.attn_cache_append.restype = _i
_lib.attn_cache_fwd.argtypes = [_vp] * 11 + [_sz] + [_i] * 7 + [_f, _vp]
_lib.attn_cache_fwd.restype = _i
_lib.attn_cache_fwd_workspace_bytes.argtypes = [_i] * 6
_lib.attn_cache_fwd_workspace_bytes.restype = _sz
_lib.attn_cache_weights.argtypes = [_vp] * 9 + [_i] * 7 + [_f, _vp]
_lib.attn_cache_weights.restype = _i
_lib.attn_cache_evict.argtypes = [_vp] * 12 + [_i] * 7 + [_vp]
_lib.attn_cache_evict.restype = _i
_lib.attn_status_string.argtypes = [_i]
_lib.attn_status_string.restype = ctypes.c_char_p
_lib.attn_fwd_key_tile.argtypes = [_i]
_lib.attn_fwd_key_tile.restype = _i

FWD_SINGLE_ROUNDING = 1
FWD_PV_E4M3 = 2
FWD_GUARD_UNDERFLOW = 4

EXPORTS = ["attn_fwd", "attn_fwd_ex", "attn_fwd_opt", "attn_delta", "attn_delta_hp",
           "attn_delta_recompute", "attn_bwd", "attn_bwd_noalloc", "attn_bwd_noalloc_max_rows",
           "attn_bwd_dkdv", "attn_bwd_dq", "attn_bwd_dq_delta", "attn_fwd_strided", "attn_bwd_strided",
           "attn_fwd_gqa", "attn_bwd_gqa", "attn_fwd_rect", "attn_bwd_rect",
           "attn_bwd_workspace_bytes", "attn_fwd_ws", "attn_fwd_workspace_bytes",
           "attn_status_string", "attn_fwd_key_tile", "attn_rope", "attn_rope_frequencies", "attn_cache_append",
           "attn_cache_fwd", "attn_cache_fwd_workspace_bytes", "attn_cache_weights", "attn_cache_evict"]


class AttnError(RuntimeError):
    def __init__(self, status):
        self.status = int(status)
        super().__init__(_lib.attn_status_string(int(status)).decode())


def raw():
    """The ctypes library object (for tests that call the C ABI with hand-made arguments)."""
    return _lib


def status_string(status):
    return _lib.attn_status_string(int(status)).decode()


def fwd_key_tile(d):
    return int(_lib.attn_fwd_key_tile(int(d)))


def bwd_workspace_bytes(B, H, N, d):
    return int(_lib.attn_bwd_workspace_bytes(B, H, N, d))


def _check(status):
    if status != 0:
        raise AttnError(status)


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def _bhnd(t, name):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor [B,H,N,d]")
    return t.shape


# below, the library wants no workspace whatever the grid: not worth asking (1 us of host time in a 12 us call)
_MIN_SHARED_KEYS = 1024


def fwd_workspace_bytes(B, H, Nq, Nk, d, causal, variant=STANDARD):
    """Workspace the forward can use for this problem (0: none, one pass over the keys is as fast)."""
    return int(_lib.attn_fwd_workspace_bytes(B, H, Nq, Nk, d, int(bool(causal)), int(variant)))


def _fwd_shared_out(Q, K, V, O, LSE, strides, H_kv, Nk, causal, softmax_scale, variant, beta, eps, stream,
                    workspace, allocate):
    """attn_fwd_ws of the C ABI where the library wants a workspace for this problem (grids of few
    query blocks) and there is one, the caller's or (`allocate`) a new one; False, and nothing done, otherwise."""
    if Nk < _MIN_SHARED_KEYS or (workspace is None and not allocate):
        return False
    B, H, N, d = Q.shape
    need = fwd_workspace_bytes(B, H, N, Nk, d, causal, variant)
    if need == 0:
        return False
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor")
        need = workspace.numel() * workspace.element_size()
    elif stream is not None and stream != torch.cuda.current_stream():
        with torch.cuda.stream(stream):          # the workspace belongs to the stream that uses it
            workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
    else:
        workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
    _check(_lib.attn_fwd_ws(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(workspace), need, *strides, B, H, H_kv,
                            N, Nk, d, int(bool(causal)), float(softmax_scale), int(variant),
                            float(DEFAULT_BETA if beta is None else beta),
                            float(DEFAULT_EPS if eps is None else eps), _stream(stream)))
    return True


def attn_fwd(Q, K, V, causal, softmax_scale, variant=STANDARD, beta=None, eps=None,
             O=None, LSE=None, stream=None, workspace=None, one_pass=False):
    """O, LSE = attention forward: attn_fwd_ws of the C ABI where few query blocks meet many keys
    (fwd_workspace_bytes(...) > 0), attn_fwd / attn_fwd_ex otherwise.  The two add the same terms in
    another float32 order (a bf16 step in a few of 10^4 elements of O).

    workspace: a CUDA tensor of at least fwd_workspace_bytes(...) bytes; one is allocated when absent, unless
    both O and LSE are given: such a call allocates nothing and runs the one-pass kernel.
    one_pass: the one-pass kernel (that of attn_fwd_opt, bit for bit) in any case."""
    B, H, N, d = _bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    allocate = O is None or LSE is None
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None:
        LSE = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    if not one_pass and _fwd_shared_out(Q, K, V, O, LSE, (0, 0, 0), H, N, causal, softmax_scale, variant, beta, eps,
                                        stream, workspace, allocate):
        return O, LSE
    if beta is None and eps is None:
        st = _lib.attn_fwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), B, H, N, d, int(bool(causal)),
                           float(softmax_scale), int(variant), _stream(stream))
    else:
        st = _lib.attn_fwd_ex(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), B, H, N, d, int(bool(causal)),
                              float(softmax_scale), int(variant),
                              float(DEFAULT_BETA if beta is None else beta),
                              float(DEFAULT_EPS if eps is None else eps), _stream(stream))
    _check(st)
    return O, LSE


def attn_fwd_opt(Q, K, V, causal, softmax_scale, variant=STANDARD, beta=None, eps=None,
                 want_O_hp=False, want_counts=False, single_rounding=False, pv_e4m3=False,
                 guard_underflow=False, O=None, LSE=None, stream=None):
    """attn_fwd_opt of the C ABI: returns a dict with O, LSE and, when asked for, O_hp (float32
    [B,H,N,d]), ones and fired (int32 [B,H,N])."""
    B, H, N, d = _bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    out = {"O": torch.empty_like(Q) if O is None else O,
           "LSE": torch.empty((B, H, N), dtype=torch.float32, device=Q.device) if LSE is None else LSE}
    if want_O_hp:
        out["O_hp"] = torch.empty((B, H, N, d), dtype=torch.float32, device=Q.device)
    if want_counts:
        out["ones"] = torch.empty((B, H, N), dtype=torch.int32, device=Q.device)
        out["fired"] = torch.empty((B, H, N), dtype=torch.int32, device=Q.device)
    opt = lambda k: _ptr(out[k]) if k in out else None
    st = _lib.attn_fwd_opt(_ptr(Q), _ptr(K), _ptr(V), _ptr(out["O"]), _ptr(out["LSE"]), opt("O_hp"),
                           opt("ones"), opt("fired"), B, H, N, d, int(bool(causal)),
                           float(softmax_scale), int(variant),
                           float(DEFAULT_BETA if beta is None else beta),
                           float(DEFAULT_EPS if eps is None else eps),
                           (FWD_SINGLE_ROUNDING if single_rounding else 0) | (FWD_PV_E4M3 if pv_e4m3 else 0)
                           | (FWD_GUARD_UNDERFLOW if guard_underflow else 0),
                           _stream(stream))
    _check(st)
    return out


def attn_delta_hp(O_hp, dO, delta=None, stream=None):
    """delta_hp = rowsum(dO o O_hp), float32 [B,H,N], from the float32 O_hp of attn_fwd_opt."""
    B, H, N, d = _bhnd(dO, "dO")
    if O_hp.dtype != torch.float32 or not O_hp.is_cuda or not O_hp.is_contiguous() or tuple(O_hp.shape) != (B, H, N, d):
        raise ValueError("O_hp must be a contiguous CUDA float32 tensor shaped like dO")
    if delta is None:
        delta = torch.empty((B, H, N), dtype=torch.float32, device=dO.device)
    _check(_lib.attn_delta_hp(_ptr(O_hp), _ptr(dO), _ptr(delta), B, H, N, d, _stream(stream)))
    return delta


def attn_delta_recompute(Q, K, V, dO, LSE, causal, softmax_scale, delta=None, stream=None):
    """delta = rowsum(P o dP), recomputed in float32 from Q, K, V, dO and LSE."""
    B, H, N, d = _bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V), ("dO", dO)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    if delta is None:
        delta = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    _check(_lib.attn_delta_recompute(_ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(LSE), _ptr(delta),
                                     B, H, N, d, int(bool(causal)), float(softmax_scale),
                                     _stream(stream)))
    return delta


def attn_delta(O, dO, delta=None, stream=None):
    """delta = rowsum(dO o O), float32 [B,H,N]."""
    B, H, N, d = _bhnd(O, "O")
    if _bhnd(dO, "dO") != (B, H, N, d):
        raise ValueError("dO shape differs from O")
    if delta is None:
        delta = torch.empty((B, H, N), dtype=torch.float32, device=O.device)
    _check(_lib.attn_delta(_ptr(O), _ptr(dO), _ptr(delta), B, H, N, d, _stream(stream)))
    return delta


def attn_bwd(Q, K, V, O, dO, LSE, causal, softmax_scale, variant=STANDARD,
             dQ=None, dK=None, dV=None, workspace=None, stream=None):
    """dQ, dK, dV = attention backward.  `workspace` (uint8 CUDA tensor) is allocated when absent;
    after the call its first B*H*N float32 hold delta."""
    B, H, N, d = _bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V), ("O", O), ("dO", dO)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(Q) if dK is None else dK
    dV = torch.empty_like(Q) if dV is None else dV
    need = bwd_workspace_bytes(B, H, N, d)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=Q.device)
    st = _lib.attn_bwd(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ), _ptr(dK),
                       _ptr(dV), _ptr(workspace), workspace.numel(), B, H, N, d, int(bool(causal)),
                       float(softmax_scale), int(variant), _stream(stream))
    _check(st)
    return dQ, dK, dV


def attn_bwd_noalloc(Q, K, V, O, dO, LSE, causal, softmax_scale, dQ, dK, dV, variant=STANDARD, stream=None):
    """attn_bwd_noalloc of the C ABI: attn_bwd with delta in the library's own device array.  The
    outputs are the caller's (this wrapper allocates nothing either)."""
    B, H, N, d = _bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V), ("O", O), ("dO", dO), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    _check(_lib.attn_bwd_noalloc(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ), _ptr(dK),
                                 _ptr(dV), B, H, N, d, int(bool(causal)), float(softmax_scale), int(variant),
                                 _stream(stream)))
    return dQ, dK, dV


def attn_bwd_dkdv(Q, K, V, dO, LSE, delta, causal, softmax_scale, dK=None, dV=None, stream=None):
    """Stage 2 of the backward pass alone: dK, dV (delta from attn_delta)."""
    B, H, N, d = _bhnd(Q, "Q")
    dK = torch.empty_like(Q) if dK is None else dK
    dV = torch.empty_like(Q) if dV is None else dV
    _check(_lib.attn_bwd_dkdv(_ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(LSE), _ptr(delta), _ptr(dK),
                              _ptr(dV), B, H, N, d, int(bool(causal)), float(softmax_scale),
                              _stream(stream)))
    return dK, dV


def attn_bwd_dq(Q, K, V, dO, LSE, delta, causal, softmax_scale, dQ=None, stream=None):
    """Stage 3 of the backward pass alone: dQ (delta from attn_delta)."""
    B, H, N, d = _bhnd(Q, "Q")
    dQ = torch.empty_like(Q) if dQ is None else dQ
    _check(_lib.attn_bwd_dq(_ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(LSE), _ptr(delta), _ptr(dQ),
                            B, H, N, d, int(bool(causal)), float(softmax_scale), _stream(stream)))
    return dQ


def attn_bwd_dq_delta(Q, K, V, O, dO, LSE, causal, softmax_scale, dQ=None, delta=None, stream=None):
    """First stage of attn_bwd: dQ, and delta = rowsum(dO o O) formed on the way (returned too)."""
    B, H, N, d = _bhnd(Q, "Q")
    dQ = torch.empty_like(Q) if dQ is None else dQ
    if delta is None:
        delta = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    _check(_lib.attn_bwd_dq_delta(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ),
                                  _ptr(delta), B, H, N, d, int(bool(causal)), float(softmax_scale),
                                  _stream(stream)))
    return dQ, delta


def _strided_bhnd(t, name, like=None):
    """A CUDA bfloat16 tensor of logical shape [B,H,N,d] with a contiguous last dimension and any
    batch / head / row strides (e.g. a permuted view of a [B,N,H,d] buffer)."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 4 or t.stride(3) != 1:
        raise ValueError(f"{name} must be a CUDA bfloat16 tensor [B,H,N,d] whose last dimension is contiguous")
    if like is not None and (t.shape != like.shape or t.stride() != like.stride()):
        raise ValueError(f"{name} must have the shape and strides of Q")
    return t.shape, t.stride()


def attn_fwd_strided(Q, K, V, causal, softmax_scale, variant=STANDARD, beta=None, eps=None,
                     O=None, LSE=None, stream=None, workspace=None, one_pass=False):
    """attn_fwd_strided of the C ABI.  Q, K, V (and O, when given) share one set of strides;
    O defaults to a tensor laid out like Q.  workspace, one_pass: as in attn_fwd."""
    (B, H, N, d), (sb, sh, sn, _) = _strided_bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V)):
        _strided_bhnd(t, n, Q)
    allocate = O is None or LSE is None
    O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device) if O is None else O
    _strided_bhnd(O, "O", Q)
    if LSE is None:
        LSE = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    # an expanded dimension (stride 0) is for attn_fwd_strided to refuse: to attn_fwd_ws three zeros mean contiguous
    if not one_pass and min(sb, sh, sn) > 0 and _fwd_shared_out(Q, K, V, O, LSE, (sb, sh, sn), H, N, causal, softmax_scale,
                                                                variant, beta, eps, stream, workspace, allocate):
        return O, LSE
    _check(_lib.attn_fwd_strided(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), sb, sh, sn, B, H, N, d,
                                 int(bool(causal)), float(softmax_scale), int(variant),
                                 float(DEFAULT_BETA if beta is None else beta),
                                 float(DEFAULT_EPS if eps is None else eps), _stream(stream)))
    return O, LSE


def attn_bwd_strided(Q, K, V, O, dO, LSE, causal, softmax_scale, variant=STANDARD,
                     dQ=None, dK=None, dV=None, workspace=None, stream=None):
    """attn_bwd_strided of the C ABI; every bf16 tensor shares Q's strides."""
    (B, H, N, d), (sb, sh, sn, _) = _strided_bhnd(Q, "Q")
    for n, t in (("K", K), ("V", V), ("O", O), ("dO", dO)):
        _strided_bhnd(t, n, Q)
    new = lambda: torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device)
    dQ = new() if dQ is None else dQ
    dK = new() if dK is None else dK
    dV = new() if dV is None else dV
    for n, t in (("dQ", dQ), ("dK", dK), ("dV", dV)):
        _strided_bhnd(t, n, Q)
    need = bwd_workspace_bytes(B, H, N, d)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=Q.device)
    _check(_lib.attn_bwd_strided(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ),
                                 _ptr(dK), _ptr(dV), _ptr(workspace), workspace.numel(), sb, sh, sn,
                                 B, H, N, d, int(bool(causal)), float(softmax_scale), int(variant),
                                 _stream(stream)))
    return dQ, dK, dV


def attn_fwd_gqa(Q, K, V, causal, softmax_scale, variant=STANDARD, beta=None, eps=None, stream=None,
                 workspace=None, one_pass=False):
    """Grouped-query forward: Q [B,H,N,d], K and V [B,H_kv,N,d] (contiguous).
    workspace, one_pass: as in attn_fwd."""
    B, H, N, d = _bhnd(Q, "Q")
    Bk, Hkv, Nk, dk = _bhnd(K, "K")
    if _bhnd(V, "V") != K.shape or (Bk, Nk, dk) != (B, N, d):
        raise ValueError("K and V must be [B,H_kv,N,d] with the batch, length and head size of Q")
    O = torch.empty_like(Q)
    LSE = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
    if not one_pass and _fwd_shared_out(Q, K, V, O, LSE, (0, 0, 0), Hkv, N, causal, softmax_scale, variant, beta, eps,
                                        stream, workspace, True):
        return O, LSE
    _check(_lib.attn_fwd_gqa(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), B, H, Hkv, N, d,
                             int(bool(causal)), float(softmax_scale), int(variant),
                             float(DEFAULT_BETA if beta is None else beta),
                             float(DEFAULT_EPS if eps is None else eps), _stream(stream)))
    return O, LSE


def attn_bwd_gqa(Q, K, V, O, dO, LSE, causal, softmax_scale, variant=STANDARD, workspace=None, stream=None):
    """Grouped-query backward: dQ like Q, dK and dV like K."""
    B, H, N, d = _bhnd(Q, "Q")
    Hkv = _bhnd(K, "K")[1]
    for n, t in (("O", O), ("dO", dO)):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape differs from Q")
    if _bhnd(V, "V") != K.shape:
        raise ValueError("V shape differs from K")
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(K)
    need = bwd_workspace_bytes(B, H, N, d)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=Q.device)
    _check(_lib.attn_bwd_gqa(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ), _ptr(dK),
                             _ptr(dV), _ptr(workspace), workspace.numel(), B, H, Hkv, N, d,
                             int(bool(causal)), float(softmax_scale), int(variant), _stream(stream)))
    return dQ, dK, dV


def attn_fwd_rect(Q, K, V, causal, softmax_scale, variant=STANDARD, beta=None, eps=None, stream=None,
                  workspace=None, one_pass=False):
    """Forward with different numbers of queries and keys: Q [B,H,Nq,d], K and V [B,H,Nk,d]
    (contiguous); the causal mask is aligned at the bottom right.  workspace, one_pass: as in attn_fwd."""
    B, H, Nq, d = _bhnd(Q, "Q")
    Bk, Hk, Nk, dk = _bhnd(K, "K")
    if _bhnd(V, "V") != K.shape or (Bk, Hk, dk) != (B, H, d):
        raise ValueError("K and V must be [B,H,Nk,d] with the batch, heads and head size of Q")
    O = torch.empty_like(Q)
    LSE = torch.empty((B, H, Nq), dtype=torch.float32, device=Q.device)
    if not one_pass and _fwd_shared_out(Q, K, V, O, LSE, (0, 0, 0), H, Nk, causal, softmax_scale, variant, beta, eps,
                                        stream, workspace, True):
        return O, LSE
    _check(_lib.attn_fwd_rect(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), B, H, Nq, Nk, d,
                              int(bool(causal)), float(softmax_scale), int(variant),
                              float(DEFAULT_BETA if beta is None else beta),
                              float(DEFAULT_EPS if eps is None else eps), _stream(stream)))
    return O, LSE


def attn_bwd_rect(Q, K, V, O, dO, LSE, causal, softmax_scale, variant=STANDARD, workspace=None, stream=None):
    """Backward of attn_fwd_rect: dQ like Q, dK and dV like K."""
    B, H, Nq, d = _bhnd(Q, "Q")
    Nk = _bhnd(K, "K")[2]
    for n, t in (("O", O), ("dO", dO)):
        if _bhnd(t, n) != (B, H, Nq, d):
            raise ValueError(f"{n} shape differs from Q")
    if _bhnd(V, "V") != K.shape or tuple(K.shape) != (B, H, Nk, d):
        raise ValueError("K and V must be [B,H,Nk,d] with the batch, heads and head size of Q")
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(K)
    need = bwd_workspace_bytes(B, H, Nq, d)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=Q.device)
    _check(_lib.attn_bwd_rect(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(LSE), _ptr(dQ), _ptr(dK),
                              _ptr(dV), _ptr(workspace), workspace.numel(), B, H, Nq, Nk, d,
                              int(bool(causal)), float(softmax_scale), int(variant), _stream(stream)))
    return dQ, dK, dV


# ---- rotary positions and the 8-bit cache

try:
    from . import _operators            # plain calls, marshalled in C++; None (False) from it: not a plain call, handled here
except ImportError as e:
    class _Missing:
        """Attention needs nothing of it: the calls that do raise."""
        def __init__(self, cause):
            self.cause = cause

        def __getattr__(self, name):
            raise ImportError("the plain calls' marshalling is missing or does not fit this torch: build it with "
                              "`python -m paper_2510_04212_amd.build`") from self.cause

    _operators = _Missing(e)

_PLAIN = (torch.Tensor, torch.nn.Parameter)
CACHE_BLOCK = 64
_ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_length=0, beta_fast=32.0, beta_slow=1.0, device=None):
    """(frequencies, magnitude) for attn_rope: a float64 tensor [rot/2] of radians per position on `device` (default: the current GPU),
    and the factor on the rotated values (1 except under "yarn").  scaling: "none", "linear", "ntk" or "yarn", as attn_rope_frequencies of
    the C ABI describes them."""
    if scaling not in _ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {', '.join(_ROPE_SCALINGS)}")
    _fit(int(rot))
    out = torch.empty(min(max(int(rot) // 2, 1), 128), dtype=torch.float64)          # (rot above 256 is refused)
    magnitude = ctypes.c_float()
    _check(_lib.attn_rope_frequencies(_ptr(out), ctypes.byref(magnitude), int(rot), float(base), _ROPE_SCALINGS[scaling], float(factor),
                                      float(original_length), float(beta_fast), float(beta_slow)))
    return out.to("cuda" if device is None else device), magnitude.value


def _on(device, stream, make):
    """make() with the stream that the call will run on as the current one: its memory belongs to that stream."""
    if stream is None or stream == torch.cuda.current_stream(device):
        return make()
    with torch.cuda.stream(stream):
        return make()


def _fit(*sizes):
    """Checks sizes that the C ABI takes as int (ctypes would cut them)."""
    if any(not -2 ** 31 <= s < 2 ** 31 for s in sizes):
        raise ValueError(f"sizes must be below 2^31: {sizes}")


def _rows(t, name):
    """Checks a CUDA bfloat16 tensor [B,H,N,d] on the current GPU with a contiguous last dimension; any other strides."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] > 1):
        raise ValueError(f"{name} must be a CUDA bfloat16 tensor [B,H,N,d] whose last dimension is contiguous")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current GPU")
    _fit(*t.shape)
    return t.shape


def _dense(t, name, shape, dtype, device):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on {device}")
    return t


def _strides(*tensors):
    """The host array of stride_b, stride_h, stride_n of each tensor; None where all are contiguous.  The stride of a dimension of one is
    whatever torch says, and never used: the contiguous one, or 0, goes in its place."""
    if all(t is None or t.is_contiguous() for t in tensors):
        return None
    out = []
    for t in tensors:
        if t is None:
            out += [0, 0, 0]
        elif t.is_contiguous():
            B, H, N, d = t.shape
            out += [H * N * d, N * d, d]
        else:
            out += [t.stride(i) if t.shape[i] > 1 else 8 * max(1, (t.shape[3] + 7) // 8) for i in range(3)]
    return (ctypes.c_longlong * len(out))(*out)


def _ptr_or_none(t):
    """NULL for an absent argument.  A tensor subclass that has its data elsewhere has that address, too: it is not absent."""
    if t is None:
        return None
    if t.data_ptr() == 0 and t.numel() > 0:
        raise ValueError(f"a {type(t).__name__} without memory of its own cannot be passed on")
    return ctypes.c_void_p(t.data_ptr())


def attn_rope(Q, K=None, frequencies=None, positions=None, interleaved=False, magnitude=1.0, inverse=False, Q_out=None, K_out=None,
              stream=None):
    """Q_out, K_out (None without K): the first 2 * len(frequencies) columns of queries and keys rotated by their positions.

    Q [B,H,N,d], K [B,H_kv,N,d] with any strides; frequencies: rope_frequencies(...)[0]; positions: int32 [N] or [B,N], the default 0 .. N-1.
    Outputs are new tensors laid out like the inputs, or Q_out, K_out, which may be Q and K themselves.  inverse: rotates back, which is the
    backward pass (autograd.rope has both)."""
    if Q_out is None and K_out is None and stream is None and type(Q) in _PLAIN and frequencies is not None:
        out = _operators.rope(Q, K, frequencies, positions, interleaved, magnitude, inverse)
        if out is not None:
            return out
    B, H, N, d = _rows(Q, "Q")
    device = Q.device
    H_kv = 0
    if K is not None:
        H_kv = _rows(K, "K")[1]
        if (K.shape[0], K.shape[2], K.shape[3]) != (B, N, d):
            raise ValueError("K must be [B,H_kv,N,d] with the batch, length and head size of Q")
    if frequencies is None or frequencies.dim() != 1:
        raise ValueError("frequencies must be a float64 tensor [rot/2]")
    _dense(frequencies, "frequencies", frequencies.shape, torch.float64, device)
    _fit(2 * frequencies.shape[0])
    positions_stride = 0
    if positions is not None:
        if positions.dim() not in (1, 2) or positions.shape[-1] != N or (positions.dim() == 2 and positions.shape[0] != B) \
                or positions.dtype != torch.int32 or positions.device != device or (positions.stride(-1) != 1 and N > 1):
            raise ValueError(f"positions must be an int32 tensor [N] or [B,N] on {device} whose last dimension is contiguous")
        positions_stride = positions.stride(0) if positions.dim() == 2 and B > 1 else 0
    if Q_out is None:
        Q_out = _on(device, stream, lambda: torch.empty_like(Q))
    if K is not None and K_out is None:
        K_out = _on(device, stream, lambda: torch.empty_like(K))
    for t, like, n in ((Q_out, Q, "Q_out"), (K_out, K, "K_out")):
        if (t is None) != (like is None) or (t is not None and _rows(t, n) != like.shape):
            raise ValueError(f"{n} must have the shape of {n[0]}")
    if B and H + H_kv:
        _check(_lib.attn_rope(_ptr(Q), _ptr_or_none(K), _ptr(Q_out), _ptr_or_none(K_out), _strides(Q, K, Q_out, K_out),
                              _ptr_or_none(positions), positions_stride, _ptr(frequencies), B, H, H_kv, N, d, 2 * frequencies.shape[0],
                              int(bool(interleaved)), float(magnitude), int(bool(inverse)), _stream(stream)))
    return Q_out, K_out


class Cache(NamedTuple):
    """Keys and values of one layer in 8 bits (the layout is described in include/attn.h): K [B,H_kv,capacity,d] and V
    [B,H_kv,capacity/64,d,64] in torch.float8_e4m3fn, K_scale and V_scale float32 [B,H_kv,capacity/64] (V_scale negative: a NaN in the block)."""
    K: torch.Tensor
    V: torch.Tensor
    K_scale: torch.Tensor
    V_scale: torch.Tensor


def cache_empty(B, H_kv, capacity, d, device=None):
    """A Cache with room for `capacity` tokens (a multiple of 64) of each sequence and head; its contents are not initialised."""
    if capacity <= 0 or capacity % CACHE_BLOCK:
        raise ValueError(f"capacity must be a positive multiple of {CACHE_BLOCK}")
    new = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device="cuda" if device is None else device)
    nb = capacity // CACHE_BLOCK
    return Cache(new(torch.float8_e4m3fn, B, H_kv, capacity, d), new(torch.float8_e4m3fn, B, H_kv, nb, d, CACHE_BLOCK),
                 new(torch.float32, B, H_kv, nb), new(torch.float32, B, H_kv, nb))


def _cache_shape(cache, name="cache"):
    B, H_kv, capacity, d = cache.K.shape
    device = cache.K.device
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current GPU")
    _fit(capacity)
    nb = capacity // CACHE_BLOCK
    _dense(cache.K, name + ".K", (B, H_kv, nb * CACHE_BLOCK, d), torch.float8_e4m3fn, device)
    _dense(cache.V, name + ".V", (B, H_kv, nb, d, CACHE_BLOCK), torch.float8_e4m3fn, device)
    _dense(cache.K_scale, name + ".K_scale", (B, H_kv, nb), torch.float32, device)
    _dense(cache.V_scale, name + ".V_scale", (B, H_kv, nb), torch.float32, device)
    return B, H_kv, capacity, d, device


def _sequence_lengths(lengths, counts, B, device):
    _dense(lengths, "lengths", (B,), torch.int32, device)
    if counts is not None:
        _dense(counts, "counts", (B,), torch.int32, device)


def attn_cache_append(cache, K, V, lengths, counts=None, stream=None):
    """Quantises the new tokens K, V [B,H_kv,N,d] (any strides) into the cache, in place.

    lengths: int32 [B], the tokens of each sequence in its cache, the new ones among them; counts: int32 [B], how many of the N tokens (the
    first ones) a sequence really has; all where absent.  Tokens at positions past the capacity are not stored (lengths are on the device, and
    nothing is reported)."""
    if stream is None and _operators.cache_append(*cache, K, V, lengths, counts):
        return
    B, H_kv, capacity, d, device = _cache_shape(cache)
    if _rows(K, "K") != _rows(V, "V") or (K.shape[0], K.shape[1], K.shape[3]) != (B, H_kv, d):
        raise ValueError("K and V must be [B,H_kv,N,d] with the sequences, heads and head size of the cache")
    _sequence_lengths(lengths, counts, B, device)
    _check(_lib.attn_cache_append(_ptr(K), _ptr(V), _strides(K, V), _ptr(cache.K), _ptr(cache.V), _ptr(cache.K_scale), _ptr(cache.V_scale),
                                  _ptr(lengths), _ptr_or_none(counts), B, H_kv, K.shape[2], d, capacity, _stream(stream)))


def cache_fwd_workspace_bytes(B, H, H_kv, N, d, capacity):
    """Workspace that attn_cache_fwd needs for this problem (0: none)."""
    _fit(B, H, H_kv, N, d, capacity)
    return int(_lib.attn_cache_fwd_workspace_bytes(B, H, H_kv, N, d, capacity))


def _queries(Q, cache, name="Q"):
    B, H_kv, capacity, d, device = _cache_shape(cache)
    _, H, N, _ = _rows(Q, name)
    if (Q.shape[0], Q.shape[3]) != (B, d):
        raise ValueError(f"{name} must be [B,H,N,d] with the sequences and head size of the cache")
    return B, H, H_kv, N, d, capacity, device


def attn_cache_fwd(Q, cache, lengths, softmax_scale, causal=True, counts=None, O=None, LSE=None, workspace=None, stream=None):
    """O, LSE = attention of the newest queries Q [B,H,N,d] (any strides) over the cache, their own tokens appended before: query i of
    sequence b sees the first lengths[b] - counts[b] + i + 1 tokens (all lengths[b] without causal); one that sees nothing, or i >=
    counts[b], gives O = 0 and LSE = -infinity.  lengths, counts: as in attn_cache_append.

    workspace: a CUDA tensor of at least cache_fwd_workspace_bytes(...) bytes; allocated when absent.  Calls that may overlap in time (two
    streams, two graphs) need one each."""
    if O is None and LSE is None and workspace is None and stream is None:
        out = _operators.cache_fwd(*cache, Q, lengths, softmax_scale, causal, counts)
        if out is not None:
            return out
    B, H, H_kv, N, d, capacity, device = _queries(Q, cache)
    _sequence_lengths(lengths, counts, B, device)
    if O is None:
        O = _on(device, stream, lambda: torch.empty((B, H, N, d), dtype=Q.dtype, device=device))
    elif _rows(O, "O") != Q.shape:
        raise ValueError("O must have the shape of Q")
    if LSE is None:
        LSE = _on(device, stream, lambda: torch.empty((B, H, N), dtype=torch.float32, device=device))
    else:
        _dense(LSE, "LSE", (B, H, N), torch.float32, device)
    need = cache_fwd_workspace_bytes(B, H, H_kv, N, d, capacity)
    if workspace is not None:
        if not workspace.is_contiguous() or workspace.device != device:
            raise ValueError(f"workspace must be a contiguous tensor on {device}")
        need = workspace.numel() * workspace.element_size()
    elif need > 0:
        workspace = _on(device, stream, lambda: torch.empty(need, dtype=torch.uint8, device=device))
    _check(_lib.attn_cache_fwd(_ptr(Q), _strides(Q, O), _ptr(cache.K), _ptr(cache.V), _ptr(cache.K_scale), _ptr(cache.V_scale),
                               _ptr(lengths), _ptr_or_none(counts), _ptr(O), _ptr(LSE), _ptr_or_none(workspace), need, B, H, H_kv, N, d,
                               capacity, int(bool(causal)), float(softmax_scale), _stream(stream)))
    return O, LSE


def attn_cache_weights(Q, cache, LSE, lengths, softmax_scale, causal=True, counts=None, weights=None, out=None, stream=None):
    """The attention weight each cached token got from the queries of an attn_cache_fwd call (same Q, cache, lengths, softmax_scale, causal,
    counts; LSE its result), summed over those queries and the heads that share the token, added to `weights`: float32 [B,H_kv,capacity].

    weights: what tokens got before (the call's own tokens had none: not read for them); None: nothing.  out: where the result goes, `weights`
    itself for instance; a new tensor when absent.  Positions past a sequence's end become 0."""
    if stream is None:
        result = _operators.cache_weights(*cache, Q, LSE, lengths, softmax_scale, causal, counts, weights, out)
        if result is not None:
            return result if out is None else out
    B, H, H_kv, N, d, capacity, device = _queries(Q, cache)
    if H == 0 and B and H_kv:              # (the library does nothing then, and out would stay as it is)
        raise ValueError("Q must have heads")
    _sequence_lengths(lengths, counts, B, device)
    _dense(LSE, "LSE", (B, H, N), torch.float32, device)
    shape = (B, H_kv, capacity)
    if weights is not None:
        _dense(weights, "weights", shape, torch.float32, device)
    out = _on(device, stream, lambda: torch.empty(shape, dtype=torch.float32, device=device)) if out is None else \
        _dense(out, "out", shape, torch.float32, device)
    _check(_lib.attn_cache_weights(_ptr(Q), _strides(Q), _ptr(cache.K), _ptr(cache.K_scale), _ptr(LSE), _ptr(lengths), _ptr_or_none(counts),
                                   _ptr_or_none(weights), _ptr(out), B, H, H_kv, N, d, capacity, int(bool(causal)), float(softmax_scale),
                                   _stream(stream)))
    return out


def attn_cache_evict(cache, weights, lengths, budget, recent, out=None, stream=None):
    """(out, weights_out, kept): the cache cut down to min(lengths, budget) tokens of each sequence and head, the last `recent` and, of those
    before, the ones with the largest weights (equal ones: the earliest), in their order.

    weights: float32 [B,H_kv,capacity] of attn_cache_weights.  out: another Cache with room for `budget` tokens and for those that are
    to follow (one that is full takes no more); a new one of the old capacity when absent (of the budget, if that is larger).
    weights_out: float32 [B,H_kv,capacity of out], the kept tokens' weights, then 0.  kept: int32 [B,H_kv,budget], their old positions,
    then -1.  The caller's lengths are then lengths.clamp(max=budget); positions for attn_rope go on counting from the old lengths."""
    if stream is None and out is not None:
        result = _operators.cache_evict(*cache, weights, lengths, *out, budget, recent)
        if result is not None:
            return (out, *result)
    B, H_kv, capacity, d, device = _cache_shape(cache)
    _dense(weights, "weights", (B, H_kv, capacity), torch.float32, device)
    _sequence_lengths(lengths, None, B, device)
    if budget < 1:
        raise ValueError("budget must be positive")
    _fit(budget, recent)
    if out is None:
        out = _on(device, stream, lambda: cache_empty(B, H_kv, max(capacity, -(-budget // CACHE_BLOCK) * CACHE_BLOCK), d, device))
    Bo, Ho, capacity_out, do, device_out = _cache_shape(out, "out")
    if (Bo, Ho, do, device_out) != (B, H_kv, d, device):
        raise ValueError("out must have the sequences, heads and head size of the cache")
    weights_out = _on(device, stream, lambda: torch.empty((B, H_kv, capacity_out), dtype=torch.float32, device=device))
    kept = _on(device, stream, lambda: torch.empty((B, H_kv, budget), dtype=torch.int32, device=device))
    _check(_lib.attn_cache_evict(_ptr(cache.K), _ptr(cache.V), _ptr(cache.K_scale), _ptr(cache.V_scale), _ptr(weights), _ptr(lengths),
                                 _ptr(out.K), _ptr(out.V), _ptr(out.K_scale), _ptr(out.V_scale), _ptr(weights_out), _ptr(kept), B, H_kv, d,
                                 capacity, capacity_out, int(budget), int(recent), _stream(stream)))
    return out, weights_out, kept
