"""ctypes binding of libavq_attn (``include/avq_attn.h``): argument marshalling only.

Every function here hands torch device pointers and the current CUDA stream to the
C ABI; no step of the computation runs in Python or torch.  If the shared library
has not been built the first call raises - there is no CPU or torch fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libavq_attn.so")

AVQ_F32, AVQ_BF16 = 0, 1
FLAG_PARENT_STAYS, FLAG_SIMT, FLAG_CORRECTING, FLAG_CAUSAL = 1, 2, 4, 8
PROMPT_SPLIT_KEYS = 2048       # AVQ_PROMPT_SPLIT_KEYS
STATUS_NAMES = {0: "AVQ_OK", 1: "AVQ_ERR_NULL", 2: "AVQ_ERR_SHAPE", 3: "AVQ_ERR_UNSUPPORTED", 4: "AVQ_ERR_ALIGN",
                5: "AVQ_ERR_WORKSPACE", 6: "AVQ_ERR_CUDA", 7: "AVQ_ERR_DEVICE_TIMEOUT", 8: "AVQ_ERR_INDEX"}

EXPORTS = ("avq_workspace_bytes", "avq_assign", "avq_aggregate", "avq_forward", "avq_forward_host", "avq_attend",
           "avq_workspace_layout", "avq_check", "avq_status_string", "avq_version", "avq_forward_static",
           "avq_check_static", "avq_static_workspace_bytes", "avq_workspace_bytes_permuted",
           "avq_forward_permuted", "avq_codebook_update_workspace_bytes", "avq_codebook_update",
           "avq_forward_tiled", "avq_prompt_workspace_bytes", "avq_prompt_split_bytes", "avq_prompt_attend",
           "avq_prompt_attend_scratch", "avq_cache_bytes", "avq_cache_append", "avq_cache_read",
           "avq_cache_attend_workspace_bytes", "avq_cache_attend", "avq_cache_attend_scratch")


class AvqProblem(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Nq", ctypes.c_int32), ("Nk", ctypes.c_int32),
                ("d", ctypes.c_int32), ("M", ctypes.c_int32), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class AvqHeads(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class AvqCache(ctypes.Structure):
    _fields_ = [("keys", ctypes.c_void_p), ("values", ctypes.c_void_p), ("pages", ctypes.c_int32),
                ("page", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("bits", ctypes.c_int32)]


class AvqRotation(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("rows", ctypes.c_int32), ("dims", ctypes.c_int32), ("adjacent", ctypes.c_int32)]


class AvqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().avq_status_string(status).decode()
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({msg})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded shared library (loaded on first use)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_12789_b200.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        pp = ctypes.POINTER(AvqProblem)
        psz = ctypes.POINTER(ctypes.c_size_t)
        L.avq_workspace_bytes.restype, L.avq_workspace_bytes.argtypes = sz, [pp, i32, i32]
        L.avq_assign.restype, L.avq_assign.argtypes = i32, [pp, vp, vp, vp, vp, vp, vp]
        L.avq_aggregate.restype, L.avq_aggregate.argtypes = i32, [pp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.avq_forward.restype = i32
        L.avq_forward.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp]
        L.avq_forward_host.restype = i32
        L.avq_forward_host.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.avq_attend.restype = i32
        L.avq_attend.argtypes = [pp, vp, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp]
        L.avq_workspace_layout.restype = i32
        L.avq_workspace_layout.argtypes = [pp, i32, i32, psz, psz, psz, psz, psz, psz]
        L.avq_check.restype, L.avq_check.argtypes = i32, [vp, vp]
        L.avq_forward_static.restype = i32
        L.avq_forward_static.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
        L.avq_check_static.restype, L.avq_check_static.argtypes = i32, [vp]
        L.avq_static_workspace_bytes.restype, L.avq_static_workspace_bytes.argtypes = sz, []
        L.avq_workspace_bytes_permuted.restype, L.avq_workspace_bytes_permuted.argtypes = sz, [pp, i32, i32]
        L.avq_forward_permuted.restype = i32
        L.avq_forward_permuted.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.avq_forward_tiled.restype = i32
        L.avq_forward_tiled.argtypes = [pp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        L.avq_codebook_update_workspace_bytes.restype, L.avq_codebook_update_workspace_bytes.argtypes = sz, [pp]
        L.avq_codebook_update.restype = i32
        L.avq_codebook_update.argtypes = [pp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        i64, ph, pc = ctypes.c_int64, ctypes.POINTER(AvqHeads), ctypes.POINTER(AvqCache)
        L.avq_prompt_workspace_bytes.restype, L.avq_prompt_workspace_bytes.argtypes = sz, [ph]
        L.avq_prompt_split_bytes.restype, L.avq_prompt_split_bytes.argtypes = sz, [ph]
        L.avq_prompt_attend.restype = i32
        L.avq_prompt_attend.argtypes = [ph, vp, i64, vp, i64, vp, i64, vp, vp, i32, i32, i32, vp, i64, vp, vp, sz, vp]
        L.avq_prompt_attend_scratch.restype = i32
        L.avq_prompt_attend_scratch.argtypes = [*L.avq_prompt_attend.argtypes[:-3], vp, vp, sz, vp]
        L.avq_cache_bytes.restype, L.avq_cache_bytes.argtypes = sz, [pc]
        L.avq_cache_append.restype = i32
        L.avq_cache_append.argtypes = [pc, vp, i64, vp, i64, vp, i32, ctypes.POINTER(AvqRotation), vp, i64, i32, vp,
                                       i64, vp, vp]
        L.avq_cache_read.restype, L.avq_cache_read.argtypes = i32, [pc, vp, i32, vp, i64, vp, i64, vp, vp]
        L.avq_cache_attend_workspace_bytes.restype = sz
        L.avq_cache_attend_workspace_bytes.argtypes = [ph, i32, i32]
        L.avq_cache_attend.restype = i32
        L.avq_cache_attend.argtypes = [ph, pc, vp, i64, vp, i32, vp, i32, i32, vp, i64, vp, vp, sz, vp]
        L.avq_cache_attend_scratch.restype = i32
        L.avq_cache_attend_scratch.argtypes = [*L.avq_cache_attend.argtypes[:-3], vp, vp, sz, vp]
        L.avq_status_string.restype, L.avq_status_string.argtypes = ctypes.c_char_p, [i32]
        L.avq_version.restype, L.avq_version.argtypes = i32, []
        _lib = L
    return _lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return AVQ_F32
    if t.dtype == torch.bfloat16:
        return AVQ_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _raw_stream() -> int:
    """The current stream of the current device."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(_raw_stream())


def _chk(*ts: torch.Tensor) -> None:
    for t in ts:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous CUDA tensors")


def problem(B, H, Nq, Nk, d, M, C, dtype_code, scale, flags=0) -> AvqProblem:
    return AvqProblem(B, H, Nq, Nk, d, M, C, dtype_code, float(scale), flags)


def _problem_from(Q, K, Cp, Cc, scale, flags) -> AvqProblem:
    B, H, Nk, d = K.shape
    Nq = Q.shape[2] if Q is not None else Nk
    Hc, M, C, dc = Cc.shape
    if tuple(Cp.shape) != (H, M, d) or Hc != H or dc != d:
        raise ValueError("codebook shapes must be Cp [H,M,d], Cc [H,M,C,d]")
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    return problem(B, H, Nq, Nk, d, M, C, _dtype_code(K), scale, flags)


def workspace_bytes(prob: AvqProblem, P: int, block_q: int) -> int:
    return int(lib().avq_workspace_bytes(ctypes.byref(prob), P, block_q))


def assign(K, Cp, Cc, flags: int = 0):
    """avq_assign: returns (parent_idx, child_idx), int32 [B,H,Nk]."""
    _chk(K, Cp, Cc)
    prob = _problem_from(None, K, Cp, Cc, 1.0, flags)
    B, H, Nk, _ = K.shape
    pidx = torch.empty((B, H, Nk), dtype=torch.int32, device=K.device)
    cidx = torch.empty_like(pidx)
    st = lib().avq_assign(ctypes.byref(prob), _ptr(K), _ptr(Cp), _ptr(Cc), _ptr(pidx), _ptr(cidx), _stream())
    if st != 0:
        raise AvqError(st, "avq_assign")
    return pidx, cidx


def aggregate(V, parent_idx, child_idx, M: int, C: int, flags: int = 0):
    """avq_aggregate: returns (Vp [B,H,M,d], np [B,H,M], Vc [B,H,M,C,d], nc [B,H,M,C]), float32."""
    _chk(V, parent_idx, child_idx)
    B, H, Nk, d = V.shape
    prob = problem(B, H, Nk, Nk, d, M, C, _dtype_code(V), 1.0, flags)
    f32 = dict(dtype=torch.float32, device=V.device)
    Vp, n_p = torch.empty((B, H, M, d), **f32), torch.empty((B, H, M), **f32)
    Vc, n_c = torch.empty((B, H, M, C, d), **f32), torch.empty((B, H, M, C), **f32)
    st = lib().avq_aggregate(ctypes.byref(prob), _ptr(V), _ptr(parent_idx), _ptr(child_idx), _ptr(Vp), _ptr(n_p),
                             _ptr(Vc), _ptr(n_c), _stream())
    if st != 0:
        raise AvqError(st, "avq_aggregate")
    return Vp, n_p, Vc, n_c


class Forward:
    """Pre-sized buffers for repeated ``avq_forward`` calls on one problem shape."""

    def __init__(self, B, H, Nq, Nk, d, M, C, P, block_q, dtype=torch.bfloat16, scale=None, flags=0,
                 device="cuda", aux=False):
        self.P, self.block_q = P, block_q
        code = AVQ_F32 if dtype == torch.float32 else AVQ_BF16
        self.prob = problem(B, H, Nq, Nk, d, M, C, code, scale if scale is not None else 1.0 / math.sqrt(d), flags)
        nbytes = workspace_bytes(self.prob, P, block_q)
        if nbytes == 0:
            st = lib().avq_workspace_layout(ctypes.byref(self.prob), P, block_q, None, None, None, None, None, None)
            raise AvqError(st, "avq_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.nblk = (Nq + block_q - 1) // block_q
        self.topp = torch.empty((B, H, self.nblk, P), dtype=torch.int32, device=device) if aux else None
        self.importance = torch.empty((B, H, self.nblk, M), dtype=torch.float32, device=device) if aux else None
        self.dtype, self.device = dtype, device
        self.shape_y = (B, H, Nq, d)

    def __call__(self, Q, K, V, Cp, Cc, Y=None):
        _chk(Q, K, V, Cp, Cc)
        if Y is None:
            Y = torch.empty(self.shape_y, dtype=self.dtype, device=Q.device)
        # (addresses as plain integers and the problem itself, which the argument types convert: no object is made for each)
        st = (_lib or lib()).avq_forward(self.prob, Q.data_ptr(), K.data_ptr(), V.data_ptr(), Cp.data_ptr(),
                                         Cc.data_ptr(), self.P, self.block_q, Y.data_ptr(), _ptr(self.topp),
                                         _ptr(self.importance), self.workspace.data_ptr(), self.workspace.numel(),
                                         _raw_stream())
        if st != 0:
            raise AvqError(st, "avq_forward")
        return Y

    def attend(self, Q, Cp, Cc, Y=None):
        """avq_attend: stage 3 only, over the aggregates the last full call left in the workspace."""
        _chk(Q, Cp, Cc)
        if Y is None:
            Y = torch.empty(self.shape_y, dtype=self.dtype, device=Q.device)
        st = (_lib or lib()).avq_attend(self.prob, Q.data_ptr(), Cp.data_ptr(), Cc.data_ptr(), self.P, self.block_q,
                                        Y.data_ptr(), _ptr(self.topp), _ptr(self.importance), self.workspace.data_ptr(),
                                        self.workspace.numel(), _raw_stream())
        if st != 0:
            raise AvqError(st, "avq_attend")
        return Y

    def host(self, hQ, hK, hV, Cp, Cc, hY, dQ, dK, dV, dY):
        """avq_forward_host: Q, K, V, Y in (pinned) host tensors, staged through dQ..dY."""
        st = lib().avq_forward_host(ctypes.byref(self.prob), _ptr(hQ), _ptr(hK), _ptr(hV), _ptr(Cp), _ptr(Cc),
                                    self.P, self.block_q, _ptr(hY), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dY),
                                    _ptr(self.workspace), self.workspace.numel(), _stream())
        if st != 0:
            raise AvqError(st, "avq_forward_host")
        return hY

    def check(self) -> None:
        """avq_check: raises if a kernel recorded an expired device-side wait."""
        st = lib().avq_check(_ptr(self.workspace), _stream())
        if st != 0:
            raise AvqError(st, "avq_check")

    def intermediates(self):
        """Views of the indices and aggregates the last call left in the workspace."""
        offs = [ctypes.c_size_t() for _ in range(6)]
        st = lib().avq_workspace_layout(ctypes.byref(self.prob), self.P, self.block_q, *[ctypes.byref(o) for o in offs])
        if st != 0:
            raise AvqError(st, "avq_workspace_layout")
        p = self.prob
        BH = (p.B, p.H)

        def view(off, shape, dt):
            n = math.prod(shape) * 4
            return self.workspace[off.value:off.value + n].view(dt).view(*shape)

        return dict(parent_idx=view(offs[0], (*BH, p.Nk), torch.int32),
                    child_idx=view(offs[1], (*BH, p.Nk), torch.int32),
                    Vp=view(offs[2], (*BH, p.M, p.d), torch.float32), np=view(offs[3], (*BH, p.M), torch.float32),
                    Vc=view(offs[4], (*BH, p.M, p.C, p.d), torch.float32),
                    nc=view(offs[5], (*BH, p.M, p.C), torch.float32))


def forward(Q, K, V, Cp, Cc, P: int, block_q: int, scale=None, flags: int = 0, aux: bool = False):
    """One-shot avq_forward.  Returns Y, or (Y, topp, importance, intermediates) with ``aux``."""
    B, H, Nq, d = Q.shape
    Nk = K.shape[2]
    M, C = Cc.shape[1], Cc.shape[2]
    f = Forward(B, H, Nq, Nk, d, M, C, P, block_q, dtype=Q.dtype, scale=scale, flags=flags, device=Q.device,
                aux=aux)
    Y = f(Q, K, V, Cp, Cc)
    f.check()
    if aux:
        return Y, f.topp, f.importance, f.intermediates()
    return Y


def forward_permuted(Q, K, V, Cp, Cc, P: int, block_q: int, perm, scale=None, flags: int = 0):
    """avq_forward_permuted: query tiles follow ``perm`` (int32 [Nq]).  Returns (Y, topp, importance, status)
    where status is what avq_check reports after the call (0, or 8 if perm held an index out of range)."""
    _chk(Q, K, V, Cp, Cc, perm)
    prob = _problem_from(Q, K, Cp, Cc, scale, flags)
    B, H, Nq, d = Q.shape
    nblk = (Nq + block_q - 1) // block_q
    nbytes = int(lib().avq_workspace_bytes_permuted(ctypes.byref(prob), P, block_q))
    if nbytes == 0:
        raise AvqError(lib().avq_workspace_layout(ctypes.byref(prob), P, block_q, None, None, None, None, None, None)
                       or 3, "avq_workspace_bytes_permuted")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    Y = torch.zeros_like(Q)
    topp = torch.empty((B, H, nblk, P), dtype=torch.int32, device=Q.device)
    imp = torch.empty((B, H, nblk, prob.M), dtype=torch.float32, device=Q.device)
    st = lib().avq_forward_permuted(ctypes.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _ptr(Cp), _ptr(Cc), P, block_q,
                                    _ptr(perm), _ptr(Y), _ptr(topp), _ptr(imp), _ptr(ws), nbytes, _stream())
    if st != 0:
        raise AvqError(st, "avq_forward_permuted")
    return Y, topp, imp, int(lib().avq_check(_ptr(ws), _stream()))


def forward_tiled(Q, K, V, Cp, Cc, P: int, block_q: int, tile_m: int, scale=None, flags: int = 0):
    """avq_forward_tiled: selection from the tiled importance (FLAG_SIMT: CUDA-core kernels throughout).
    Returns (Y, topp, importance)."""
    _chk(Q, K, V, Cp, Cc)
    prob = _problem_from(Q, K, Cp, Cc, scale, flags | FLAG_SIMT)
    B, H, Nq, d = Q.shape
    nblk = (Nq + block_q - 1) // block_q
    nbytes = workspace_bytes(prob, P, block_q)
    if nbytes == 0:
        raise AvqError(lib().avq_workspace_layout(ctypes.byref(prob), P, block_q, None, None, None, None, None, None)
                       or 3, "avq_workspace_bytes")
    prob.flags = flags                     # (FLAG_SIMT above sizes the workspace)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=Q.device)
    Y = torch.empty_like(Q)
    topp = torch.empty((B, H, nblk, P), dtype=torch.int32, device=Q.device)
    imp = torch.empty((B, H, nblk, prob.M), dtype=torch.float32, device=Q.device)
    st = lib().avq_forward_tiled(ctypes.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _ptr(Cp), _ptr(Cc), P, block_q,
                                 tile_m, _ptr(Y), _ptr(topp), _ptr(imp), _ptr(ws), nbytes, _stream())
    if st != 0:
        raise AvqError(st, "avq_forward_tiled")
    return Y, topp, imp


def codebook_update(K, Cp, Cc, Sp, Np, Sc, Nc, decay: float, flags: int = 0):
    """avq_codebook_update: EMA statistics (updated in place) and the new codebooks (Cp', Cc')."""
    _chk(K, Cp, Cc, Sp, Np, Sc, Nc)
    prob = _problem_from(None, K, Cp, Cc, 1.0, flags)
    nbytes = int(lib().avq_codebook_update_workspace_bytes(ctypes.byref(prob)))
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=K.device)
    Cp2, Cc2 = torch.empty_like(Cp), torch.empty_like(Cc)
    st = lib().avq_codebook_update(ctypes.byref(prob), _ptr(K), _ptr(Cp), _ptr(Cc), decay, _ptr(Sp), _ptr(Np),
                                   _ptr(Sc), _ptr(Nc), _ptr(Cp2), _ptr(Cc2), _ptr(ws), ws.numel(), _stream())
    if st != 0:
        raise AvqError(st, "avq_codebook_update")
    return Cp2, Cc2


def forward_static(Q, K, V, Cp, Cc, P: int, block_q: int, scale=None, flags: int = 0, aux: bool = False):
    """avq_forward_static: the forward pass in the library's built-in scratch array, for callers
    that cannot allocate a workspace.  Only the outputs are torch tensors here; nothing else is
    allocated on the device.  Returns Y, or (Y, topp, importance) with ``aux``."""
    _chk(Q, K, V, Cp, Cc)
    prob = _problem_from(Q, K, Cp, Cc, scale, flags)
    B, H, Nq, d = Q.shape
    nblk = (Nq + block_q - 1) // block_q
    Y = torch.empty_like(Q)
    topp = torch.empty((B, H, nblk, P), dtype=torch.int32, device=Q.device) if aux else None
    imp = torch.empty((B, H, nblk, prob.M), dtype=torch.float32, device=Q.device) if aux else None
    st = lib().avq_forward_static(ctypes.byref(prob), _ptr(Q), _ptr(K), _ptr(V), _ptr(Cp), _ptr(Cc), P, block_q,
                                  _ptr(Y), _ptr(topp), _ptr(imp), _stream())
    if st != 0:
        raise AvqError(st, "avq_forward_static")
    st = lib().avq_check_static(_stream())
    if st != 0:
        raise AvqError(st, "avq_check_static")
    return (Y, topp, imp) if aux else Y


# ---------------------------------------------------------------- exact attention
# (These run at every call of a model's layer: few Python operations on the way where all is well.)
def _rows(name, t, heads, d, dtype, T):
    """A tensor of T rows, [T, heads, d] with dense heads and rows any distance apart; returns that distance."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != T or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{name} must be [{T}, {heads}, {d}], not {tuple(shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    row, head, one = t.stride()
    if T and (one != 1 or (head != d and heads > 1)):
        raise ValueError(f"the heads of a row of {name} must be dense")
    # (the stride of a single row, or of none, is anybody's: any usable one will do)
    return row if T > 1 else heads * d


def _ints(name, t, shape):
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape}, not {t.dtype} {tuple(t.shape)}")


def _here(at, *ts):
    """All tensors (None: no tensor) are on device `at`, the current one, whose current stream the call goes to."""
    for t in ts:
        if t is not None and t.get_device() != at:
            raise ValueError(f"tensors must be on the current CUDA device, not on {t.device}")


def _check(header):
    # (behind the work of the current device's stream: a header of another device would be read too early)
    _here(torch._C._cuda_getDevice() if header.is_cuda else -2, header)
    st = lib().avq_check(_ptr(header), _stream())
    if st != 0:
        raise AvqError(st, "avq_check")


def _capturing():
    return torch._C._cuda_isCurrentStreamCapturing()


_NO_LOCK = contextlib.nullcontext()                        # (a call with room of its own waits for nobody)


class _Room:
    """A plan's workspace: the header, which all of its calls share, and room for partial results.

    The room is for calls on one stream, that of the first of them, and for one thread at a time (`lock`: a call is two
    launches, and another's must not come between).  Calls on other streams and calls that are being captured take theirs
    from the allocator: its blocks are that stream's or that graph's own.  So a plan may serve any number of them at once."""
    __slots__ = ("workspace", "header", "rest", "bytes", "stream", "lock")

    def __init__(self, n, device):
        self.workspace = torch.empty(n, dtype=torch.uint8, device=device)
        self.workspace[:256].zero_()
        self.header = self.workspace.data_ptr()
        self.rest, self.bytes, self.stream, self.lock = self.header + 256, n - 256, None, threading.Lock()

    def scratch(self, stream):
        """(Under `lock`) the address of the room that a call on this stream, the current one, takes; whom to keep till then."""
        if not _capturing():
            if self.stream == stream:
                return self.rest, None
            if self.stream is None:
                self.stream = stream
                self.workspace.record_stream(torch.cuda.current_stream())
                return self.rest, None
        room = self.workspace.new_empty(self.bytes)
        return room.data_ptr(), room

    def __reduce__(self):                                  # (a copy has room and a header of its own)
        return _Room, (256 + self.bytes, self.workspace.device)


class ExactAttention:
    """avq_prompt_attend: softmax attention over packed sequences, planned for one set of heads.

    ``ExactAttention(H, Hk, d)(Q, K, V, cu_q, cu_k=None)`` takes Q [Tq,H,d], K, V [Tk,Hk,d] (rows may be views of a
    wider tensor) and the int32 bounds [S+1] of the sequences' queries and keys, and returns Y [Tq,H,d], with ``lse`` also
    the log of every query's sum, float32 [Tq,H].  ``split``: keep room (20 or 40 MB) for the parts of calls of few queries
    over many keys; calls on a second stream and captured ones take as much again for themselves.
    Rows outside all sequences are left as they are (in a Y made here: anything).  A plan has to outlive its captured graphs."""

    def __init__(self, H, Hk, d, dtype=torch.bfloat16, scale=None, causal=True, flags=0, device="cuda", split=True):
        code = {torch.float32: AVQ_F32, torch.bfloat16: AVQ_BF16}.get(dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {dtype}")
        self.heads = AvqHeads(H, Hk, d, code, float(scale) if scale is not None else 1.0 / math.sqrt(d),
                              flags | (FLAG_CAUSAL if causal else 0))
        self.dtype = dtype
        n = int((lib().avq_prompt_split_bytes if split else lib().avq_prompt_workspace_bytes)(self.heads))
        if n == 0:
            raise AvqError(lib().avq_prompt_attend(self.heads, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) or 3,
                           "avq_prompt_workspace_bytes")
        self.room, self.sizes = _Room(n, device), (H, Hk, d)
        self.workspace = self.room.workspace

    def __call__(self, Q, K, V, cu_q, cu_k=None, Y=None, lse=False):
        h, dtype = self.heads, self.dtype
        H, Hk, d = self.sizes
        Tq, Tk, S = Q.shape[0], K.shape[0], cu_q.shape[0] - 1
        if S < 0 or (cu_k is None and Tq != Tk):
            raise ValueError("cu_q must hold S + 1 bounds, and cu_k too where queries and keys differ in number")
        qs, ks, vs = (_rows("Q", Q, H, d, dtype, Tq), _rows("K", K, Hk, d, dtype, Tk), _rows("V", V, Hk, d, dtype, Tk))
        _ints("cu_q", cu_q, (S + 1,))
        if cu_k is not None:
            _ints("cu_k", cu_k, (S + 1,))
        at = torch._C._cuda_getDevice() if Q.is_cuda else -2
        _here(at, Q, K, V, cu_q, cu_k, Y, self.workspace)
        if Y is None:
            Y, ys = Q.new_empty((Tq, H, d)), H * d
        else:
            ys = _rows("Y", Y, H, d, dtype, Tq)
        L = Q.new_empty((Tq, H), dtype=torch.float32) if lse else None
        stream, room = torch._C._cuda_getCurrentRawStream(at), self.room
        with room.lock:
            if Tk < PROMPT_SPLIT_KEYS or not room.bytes:    # nothing is split: no partial results
                scratch, n = None, 0
            else:
                (scratch, kept), n = room.scratch(stream), room.bytes
            st = (_lib or lib()).avq_prompt_attend_scratch(
                h, Q.data_ptr(), qs, K.data_ptr(), ks, V.data_ptr(), vs, cu_q.data_ptr(), None if cu_k is None else cu_k.data_ptr(),
                S, Tq, Tk, Y.data_ptr(), ys, L.data_ptr() if lse else None, room.header, scratch, n, stream)
        if st != 0:
            raise AvqError(st, "avq_prompt_attend")
        return (Y, L) if lse else Y

    def __reduce__(self):
        h = self.heads
        return type(self), (h.H, h.Hk, h.d, self.dtype, h.scale, bool(h.flags & FLAG_CAUSAL), h.flags & ~FLAG_CAUSAL, self.workspace.device,
                            self.room.bytes > 0)

    def check(self) -> None:
        """avq_check: raises if a kernel left something out (unusable bounds) or gave up on a wait."""
        _check(self.workspace)


class CachePlan(tuple):
    """What ``PagedCache.plan`` makes: (heads, workspace, B, nq), and `room`, whose the workspace is."""

    def __new__(cls, heads, room, B, nq):
        plan = super().__new__(cls, (heads, room.workspace, B, nq))
        plan.room = room
        return plan

    def __reduce__(self):
        return CachePlan, (self[0], self.room, self[2], self[3])


class PagedCache:
    """A paged cache of keys and values over the caller's two buffers (avq_cache): ``append``, ``read``, ``attend``.

    ``bits``: the width of ``dtype`` for rows of that type, buffers [pages, Hk, page, d]; 4 for groups of 32 dimensions in
    4 bits, buffers uint8 [pages, Hk, page * 5 d / 8].  ``PagedCache.empty`` makes the buffers."""

    def __init__(self, keys, values, page, d, dtype=torch.bfloat16, bits=None):
        code = {torch.float32: AVQ_F32, torch.bfloat16: AVQ_BF16}.get(dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {dtype}")
        width = 32 if code == AVQ_F32 else 16
        bits = width if bits is None else bits
        pages, Hk = keys.shape[:2]
        want = ((pages, Hk, page * 5 * d // 8), torch.uint8) if bits == 4 else ((pages, Hk, page, d), dtype)
        for name, t in (("keys", keys), ("values", values)):
            if (tuple(t.shape), t.dtype) != want or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {want[1]} {want[0]}, not {t.dtype} {tuple(t.shape)}")
        if keys.device != values.device:                   # (calls look at the keys' device alone)
            raise ValueError(f"keys and values must be on one device, not on {keys.device} and {values.device}")
        self.keys, self.values, self.dtype = keys, values, dtype
        self.desc = AvqCache(keys.data_ptr(), values.data_ptr(), pages, page, Hk, d, code, bits)
        if int(lib().avq_cache_bytes(self.desc)) == 0:
            raise AvqError(lib().avq_cache_read(self.desc, 0, 0, 0, 0, 0, 0, 0, 0) or 3, "avq_cache_bytes")
        self.header = torch.zeros(256, dtype=torch.uint8, device=keys.device)
        self.sizes = (Hk, d)

    @classmethod
    def empty(cls, pages, page, Hk, d, dtype=torch.bfloat16, bits=None, device="cuda"):
        shape, dt = ((pages, Hk, page * 5 * d // 8), torch.uint8) if bits == 4 else ((pages, Hk, page, d), dtype)
        return cls(torch.zeros(shape, dtype=dt, device=device), torch.zeros(shape, dtype=dt, device=device), page, d, dtype, bits)

    def append(self, K, V, slots, pos=None, cos=None, sin=None, adjacent=False, Q=None, Q_out=None):
        """avq_cache_append: K, V [T,Hk,d] to the rows ``slots`` (int32 [T], -1: none), K rotated by the positions ``pos``
        (int32 [T]) with the float32 tables ``cos``, ``sin`` [rows, dims/2].  With Q [T,H,d] returns the rotated queries (in a
        Q_out made here the rows of slot -1 are anything)."""
        dtype, (Hk, d), T = self.dtype, self.sizes, K.shape[0]
        ks, vs = _rows("K", K, Hk, d, dtype, T), _rows("V", V, Hk, d, dtype, T)
        _ints("slots", slots, (T,))
        rot = None
        if pos is not None:
            _ints("pos", pos, (T,))
            for name, t in (("cos", cos), ("sin", sin)):
                if t is None or t.dtype is not torch.float32 or len(t.shape) != 2 or not t.is_contiguous() or t.shape != cos.shape:
                    raise ValueError(f"{name} must be a contiguous float32 table [rows, dims/2]")
            rot = AvqRotation(cos.data_ptr(), sin.data_ptr(), pos.data_ptr(), cos.shape[0], 2 * cos.shape[1], adjacent)
        elif cos is not None or sin is not None:
            raise ValueError("a rotation needs the positions")
        H = qs = os_ = 0
        if Q is not None:
            H = Q.shape[1]
            qs = _rows("Q", Q, H, d, dtype, T)
            if Q_out is None:
                Q_out, os_ = Q.new_empty((T, H, d)), H * d
            else:
                os_ = _rows("Q_out", Q_out, H, d, dtype, T)
        elif Q_out is not None:
            raise ValueError("Q_out without Q")
        at = torch._C._cuda_getDevice() if K.is_cuda else -2
        _here(at, K, V, slots, pos, cos, sin, Q, Q_out, self.keys)
        st = (_lib or lib()).avq_cache_append(self.desc, K.data_ptr(), ks, V.data_ptr(), vs, slots.data_ptr(), T, rot,
                                              None if Q is None else Q.data_ptr(), qs, H,
                                              None if Q is None else Q_out.data_ptr(), os_, self.header.data_ptr(),
                                              torch._C._cuda_getCurrentRawStream(at))
        if st != 0:
            raise AvqError(st, "avq_cache_append")
        return Q_out

    def read(self, slots, K=None, V=None):
        """avq_cache_read: the rows ``slots`` back as (K, V) [T,Hk,d]; rows of -1 are left as they are (in tensors
        made here: anything)."""
        dtype, (Hk, d), T = self.dtype, self.sizes, slots.shape[0]
        _ints("slots", slots, (T,))
        at = torch._C._cuda_getDevice() if slots.is_cuda else -2
        _here(at, slots, K, V, self.keys)
        if K is None:
            K, ks = slots.new_empty((T, Hk, d), dtype=dtype), Hk * d
        else:
            ks = _rows("K", K, Hk, d, dtype, T)
        if V is None:
            V, vs = slots.new_empty((T, Hk, d), dtype=dtype), Hk * d
        else:
            vs = _rows("V", V, Hk, d, dtype, T)
        st = (_lib or lib()).avq_cache_read(self.desc, slots.data_ptr(), T, K.data_ptr(), ks, V.data_ptr(), vs,
                                            self.header.data_ptr(), torch._C._cuda_getCurrentRawStream(at))
        if st != 0:
            raise AvqError(st, "avq_cache_read")
        return K, V

    def _heads(self, H, B, nq, scale, flags):
        """The heads of such calls, and the bytes of their workspace."""
        c = self.desc
        heads = AvqHeads(H, c.Hk, c.d, c.dtype, float(scale) if scale is not None else 1.0 / math.sqrt(c.d), flags)
        n = int(lib().avq_cache_attend_workspace_bytes(heads, B, nq))
        if n == 0:
            raise AvqError(lib().avq_cache_attend(heads, c, 0, 0, 0, 0, 0, B, nq, 0, 0, 0, 0, 0, 0) or 3,
                           "avq_cache_attend_workspace_bytes")
        return heads, n

    def plan(self, H, B, nq=1, scale=None, flags=0):
        """Workspace and heads of repeated ``attend`` calls of B sequences with nq queries each.  Calls on a second stream and
        captured ones take as much room again for themselves.  A plan has to outlive its captured graphs."""
        heads, n = self._heads(H, B, nq, scale, flags)
        return CachePlan(heads, _Room(n, self.keys.device), B, nq)

    def attend(self, Q, table, lens, scale=None, flags=0, Y=None, lse=False, plan=None):
        """avq_cache_attend: the last queries Q [B*nq,H,d] of B sequences (``lens`` int32 [B] tokens in the pages ``table``
        int32 [B, n]) over the cache.  Returns Y, or (Y, lse).  ``plan``: what ``plan`` made, its scale and flags with it (given
        here too, they have to be the same).  Without one, `check` without one tells what the call left out."""
        B = lens.shape[0]
        if plan is None:
            if B == 0 or Q.shape[0] % B:
                raise ValueError("Q must hold the same number of rows for each of the sequences of lens")
            pB, nq, room, header, lock = B, max(1, Q.shape[0] // B), None, self.header, _NO_LOCK
            heads, n = self._heads(Q.shape[1], B, nq, scale, flags)
            n, header_at = n - 256, header.data_ptr()
        elif scale is not None and ctypes.c_float(scale).value != plan[0].scale:
            raise ValueError(f"the plan's scale is {plan[0].scale}, not {scale}")
        elif flags and flags != plan[0].flags:
            raise ValueError(f"the plan's flags are {plan[0].flags}, not {flags}")
        else:
            heads, header, pB, nq = plan
            room = plan.room
            n, lock, header_at = room.bytes, room.lock, room.header
        if B != pB or len(table.shape) != 2:
            raise ValueError(f"lens must be [{pB}] and table [{pB}, n]")
        H, d, dtype, T, pages = heads.H, self.sizes[1], self.dtype, B * nq, table.shape[1]
        qs = _rows("Q", Q, H, d, dtype, T)
        _ints("lens", lens, (B,))
        _ints("table", table, (B, pages))
        at = torch._C._cuda_getDevice() if Q.is_cuda else -2
        _here(at, Q, table, lens, Y, self.keys, header)
        if Y is None:
            Y, ys = Q.new_empty((T, H, d)), H * d
        else:
            ys = _rows("Y", Y, H, d, dtype, T)
        L = Q.new_empty((T, H), dtype=torch.float32) if lse else None
        stream = torch._C._cuda_getCurrentRawStream(at)
        with lock:
            if room is None:
                kept = header.new_empty(n)
                scratch = kept.data_ptr()
            elif room.stream == stream and not _capturing():
                scratch = room.rest
            else:
                scratch, kept = room.scratch(stream)
            st = (_lib or lib()).avq_cache_attend_scratch(
                heads, self.desc, Q.data_ptr(), qs, table.data_ptr(), pages, lens.data_ptr(), B, nq, Y.data_ptr(), ys,
                L.data_ptr() if lse else None, header_at, scratch, n, stream)
        if st != 0:
            raise AvqError(st, "avq_cache_attend")
        return (Y, L) if lse else Y

    def check(self, plan=None) -> None:
        """avq_check of the cache's header (append, read, attend without a plan), or of a plan's: raises if a kernel skipped a
        slot, position, length or page out of range."""
        _check(self.header if plan is None else plan[1])
