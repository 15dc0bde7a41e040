"""ctypes binding of the MoL C ABI (include/mol.h).

Argument marshalling only: every step of the retrieval path runs in the HIP
kernels of libmol.so.  torch provides device memory and streams.  The
functions carry the C names; the lower-case helpers at the bottom allocate
outputs and workspace with torch and call them.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import numbers
import os
from typing import List, Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmol.so")

MOL_OK, MOL_EINVAL, MOL_EUNSUPPORTED, MOL_EWORKSPACE, MOL_EHIP = range(5)
MOL_F32, MOL_BF16 = 0, 1
(MOL_OP_SCORE, MOL_OP_TOPK_EXACT, MOL_OP_TOPK_PER_EMBD, MOL_OP_RERANK, MOL_OP_TOPK_MAXDOT,
 MOL_OP_TOPK_BOUNDED, MOL_OP_TOPK_TWO_PASS, MOL_OP_SCORE_GRAD) = range(8)
MOL_TWO_PASS_MIN, MOL_TWO_PASS_KTH = 0, 1
MOL_FLAG_F32_GATING = 1
MOL_FLAG_BF16X2_GATING = 2
MOL_STATE_F32, MOL_STATE_E4M3 = 0, 1
MOL_STATE_BLOCK = 256

EXPORTS = ("mol_workspace_size", "mol_score", "mol_topk_exact", "mol_topk_exact_noalloc", "mol_topk_exact_bounded",
           "mol_topk_two_pass", "mol_topk_maxdot", "mol_topk_per_embd",
           "mol_rerank", "mol_avg_embed", "mol_gap_bound", "mol_gap_bound_combined",
           "mol_embed_lookup", "mol_embed_grad_workspace", "mol_embed_grad",
           "mol_softmax_loss_workspace", "mol_softmax_loss", "mol_score_grad", "mol_adamw_step",
           "mol_timing_enable", "mol_timing_read",
           "mol_status_str", "mol_last_error")

_DTYPES = {torch.float32: MOL_F32, torch.bfloat16: MOL_BF16}


class MolError(RuntimeError):
    """A nonzero mol_status from the library."""

    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


class MolProblemC(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("Pq", ctypes.c_int32),
                ("Px", ctypes.c_int32), ("d", ctypes.c_int32), ("H", ctypes.c_int32),
                ("dtype", ctypes.c_int32),
                ("Q", ctypes.c_void_p), ("X", ctypes.c_void_p),
                ("a_q", ctypes.c_void_p), ("a_x", ctypes.c_void_p),
                ("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p),
                ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p), ("flags", ctypes.c_uint32)]


class MolScoreGradsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2")]


class MolAdamwTensorC(ctypes.Structure):
    _fields_ = ([("n", ctypes.c_int64)] +
                [(n, ctypes.c_void_p) for n in ("p", "g", "m", "v", "m_scale", "v_scale", "p_out", "m_out", "v_out",
                                                "m_scale_out", "v_scale_out", "copy_out")] +
                [("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("state", ctypes.c_int32),
                 ("weight_decay", ctypes.c_float), ("rng_offset", ctypes.c_uint64)])


class MolAdamwC(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int32), ("seed", ctypes.c_uint32),
                ("grad_scale", ctypes.c_void_p), ("lr_ptr", ctypes.c_void_p), ("step_ptr", ctypes.c_void_p)]


_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libmol.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2407_15462_amd.build` (there is no fallback)")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(MolProblemC)
    vp, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
    sig = {
        "mol_workspace_size": [P, ctypes.c_int, i32, i32, i32, ctypes.POINTER(sz)],
        "mol_score": [P, i32, i32, vp, vp],
        "mol_topk_exact": [P, i32, vp, vp, vp, sz, vp],
        "mol_topk_exact_noalloc": [P, i32, vp, vp, vp],
        "mol_topk_exact_bounded": [P, i32, vp, vp, vp, vp, sz, vp],
        "mol_topk_two_pass": [P, i32, i32, vp, vp, vp, vp, sz, vp],
        "mol_topk_maxdot": [P, i32, vp, vp, vp, sz, vp],
        "mol_topk_per_embd": [P, i32, vp, vp, vp, sz, vp],
        "mol_rerank": [P, vp, i32, vp, i32, i32, vp, vp, vp, vp, sz, vp],
        "mol_avg_embed": [P, vp, vp, vp],
        "mol_gap_bound": [i32, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp],
        "mol_gap_bound_combined": [i32, i32, i32, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp],
        "mol_embed_lookup": [vp, i32, i32, i32, i32, vp, i32, f32, vp, i32, vp],
        "mol_embed_grad_workspace": [i32, i32, i32, i32, ctypes.POINTER(sz)],
        "mol_embed_grad": [vp, i32, i32, i32, i32, vp, i32, f32, i32, vp, i32, vp, sz, vp],
        "mol_softmax_loss_workspace": [i32, i32, ctypes.POINTER(sz)],
        "mol_softmax_loss": [i32, i32, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp],
        "mol_score_grad": [P, vp, ctypes.POINTER(MolScoreGradsC), vp, sz, vp],
        "mol_adamw_step": [ctypes.POINTER(MolAdamwC), vp, i32, vp],
        "mol_timing_enable": [ctypes.c_int],
        "mol_timing_read": [ctypes.c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.mol_status_str.argtypes = [ctypes.c_int]
    lib.mol_status_str.restype = ctypes.c_char_p
    lib.mol_last_error.argtypes = []
    lib.mol_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != MOL_OK:
        lib = load()
        raise MolError(status, f"{lib.mol_status_str(status).decode()}: "
                               f"{lib.mol_last_error().decode()}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors handed to the MoL library must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())   # (a Stream object costs 5 us)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class Problem:
    """A mol_problem built from torch tensors (kept alive by this object).

    Q [B][Pq][d], X [Px][N][d] in bfloat16 or float32; a_q [B][P], a_x [N][P],
    b1 [H], b2 [P] float32; W1 [H][P], W2 [P][H] in the embedding dtype.
    Gating tensors may be None for mol_topk_per_embd.
    """

    def __init__(self, Q, X, a_q=None, a_x=None, W1=None, b1=None, W2=None, b2=None, flags: int = 0):
        self.tensors = (Q, X, a_q, a_x, W1, b1, W2, b2)
        if Q.dtype == torch.bfloat16:
            dtype = MOL_BF16
        elif Q.dtype == torch.float32:
            dtype = MOL_F32
        else:
            raise ValueError(f"unsupported embedding dtype {Q.dtype}")
        B, Pq, d = Q.shape
        Px, N, d2 = X.shape
        H = W1.shape[0] if W1 is not None else 1
        self.c = MolProblemC(B, N, Pq, Px, d if d == d2 else -1, H, dtype,
                             _ptr(Q), _ptr(X), _ptr(a_q), _ptr(a_x), _ptr(W1), _ptr(b1),
                             _ptr(W2), _ptr(b2), flags)
        self.B, self.N, self.Pq, self.Px, self.d, self.H = B, N, Pq, Px, d, H
        self.P = Pq * Px
        self.device = Q.device
        self.checked = False                   # sizes and types, which only gradients look at

    @classmethod
    def from_inputs(cls, inp, flags: int = 0) -> "Problem":
        return cls(inp.Q, inp.X, inp.a_q, inp.a_x, inp.W1, inp.b1, inp.W2, inp.b2, flags)

    @property
    def ref(self):
        return ctypes.byref(self.c)


# ---------------------------------------------------------------- C entry points
def mol_workspace_size(prob: Problem, op: int, k: int = 0, kprime: int = 0, C: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(load().mol_workspace_size(prob.ref, op, k, kprime, C, ctypes.byref(out)))
    return out.value


def mol_score(prob: Problem, n_begin: int, n_count: int, phi: torch.Tensor, stream=None) -> None:
    _check(load().mol_score(prob.ref, n_begin, n_count, _ptr(phi), _stream(stream)))


def mol_topk_exact(prob: Problem, k: int, out_score, out_idx, ws, stream=None) -> None:
    _check(load().mol_topk_exact(prob.ref, k, _ptr(out_score), _ptr(out_idx), _ptr(ws),
                                 ws.numel() if ws is not None else 0, _stream(stream)))


def mol_topk_exact_noalloc(prob: Problem, k: int, out_score, out_idx, stream=None) -> None:
    _check(load().mol_topk_exact_noalloc(prob.ref, k, _ptr(out_score), _ptr(out_idx), _stream(stream)))


def mol_topk_exact_bounded(prob: Problem, k: int, bound, out_score, out_idx, ws, stream=None) -> None:
    _check(load().mol_topk_exact_bounded(prob.ref, k, _ptr(bound), _ptr(out_score), _ptr(out_idx),
                                         _ptr(ws), ws.numel() if ws is not None else 0,
                                         _stream(stream)))


def mol_topk_two_pass(prob: Problem, k: int, mode: int, out_score, out_idx, out_bound, ws,
                      stream=None) -> None:
    _check(load().mol_topk_two_pass(prob.ref, k, mode, _ptr(out_score), _ptr(out_idx),
                                    _ptr(out_bound), _ptr(ws), ws.numel() if ws is not None else 0,
                                    _stream(stream)))


def mol_topk_maxdot(prob: Problem, k: int, out_score, out_idx, ws, stream=None) -> None:
    _check(load().mol_topk_maxdot(prob.ref, k, _ptr(out_score), _ptr(out_idx), _ptr(ws),
                                  ws.numel() if ws is not None else 0, _stream(stream)))


def mol_topk_per_embd(prob: Problem, kprime: int, out_dot, out_idx, ws, stream=None) -> None:
    _check(load().mol_topk_per_embd(prob.ref, kprime, _ptr(out_dot), _ptr(out_idx), _ptr(ws),
                                    ws.numel() if ws is not None else 0, _stream(stream)))


def mol_rerank(prob: Problem, cand, C: int, cand2, C2: int, k: int, out_score, out_idx,
               out_n_unique, ws, stream=None) -> None:
    _check(load().mol_rerank(prob.ref, _ptr(cand), C, _ptr(cand2), C2, k, _ptr(out_score),
                             _ptr(out_idx), _ptr(out_n_unique), _ptr(ws),
                             ws.numel() if ws is not None else 0, _stream(stream)))


def mol_avg_embed(prob: Problem, q_avg, x_avg, stream=None) -> None:
    _check(load().mol_avg_embed(prob.ref, _ptr(q_avg), _ptr(x_avg), _stream(stream)))


def mol_gap_bound(B: int, P: int, m: int, dots, k: int, scores, out_S, out_SK, out_bound,
                  out_looser, stream=None) -> None:
    _check(load().mol_gap_bound(B, P, m, _ptr(dots), k, _ptr(scores), _ptr(out_S), _ptr(out_SK),
                                _ptr(out_bound), _ptr(out_looser), _stream(stream)))


def mol_gap_bound_combined(B: int, P: int, m: int, dots, ids, kprime: int, avg_ids, k_avg: int, k: int,
                           scores, out_S, out_SK, out_bound, stream=None) -> None:
    _check(load().mol_gap_bound_combined(B, P, m, _ptr(dots), _ptr(ids), kprime, _ptr(avg_ids), k_avg, k,
                                         _ptr(scores), _ptr(out_S), _ptr(out_SK), _ptr(out_bound),
                                         _stream(stream)))


def _sizes(*sizes: int) -> None:
    """The library's sizes are int32: ctypes would cut others off to it."""
    if max(sizes) >= 1 << 31 or min(sizes) < -(1 << 31):
        raise ValueError(f"sizes {sizes}: the library takes up to 2^31 - 1")


def mol_embed_grad_workspace(C: int, V: int, d: int, T: int) -> int:
    _sizes(C, V, d, T)
    out = ctypes.c_size_t(0)
    _check(load().mol_embed_grad_workspace(C, V, d, T, ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=256)              # (a call of its own costs a tenth of a small loss)
def mol_softmax_loss_workspace(B: int, N: int) -> int:
    _sizes(B, N)
    out = ctypes.c_size_t(0)
    _check(load().mol_softmax_loss_workspace(B, N, ctypes.byref(out)))
    return out.value


def mol_softmax_loss(phi, target, ids, inv_temp: float, row_weight, loss, dphi, ws, stream=None) -> None:
    B, N = phi.shape
    _sizes(B, N)
    _check(load().mol_softmax_loss(B, N, _ptr(phi), _ptr(target), _ptr(ids), inv_temp, _ptr(row_weight), _ptr(loss),
                                   _ptr(dphi), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)))


def mol_adamw_step(opt: MolAdamwC, tensors, n_tensors: int, stream=None) -> None:
    _check(load().mol_adamw_step(ctypes.byref(opt), tensors, n_tensors, _stream(stream)))


def mol_timing_enable(on: bool) -> None:
    _check(load().mol_timing_enable(1 if on else 0))


def mol_timing_read(op: int) -> Tuple[float, int]:
    """(summed milliseconds, launch count) of the main kernel of ``op`` since
    the last read; waits for the recorded events."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int32(0)
    _check(load().mol_timing_read(op, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


# ------------------------------------------------- torch-allocating conveniences
def workspace(prob: Problem, op: int, k: int = 0, kprime: int = 0, C: int = 0) -> torch.Tensor:
    """A uint8 device buffer of the size the library asks for (>= 1 byte)."""
    n = mol_workspace_size(prob, op, k, kprime, C)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=prob.device)


def score(prob: Problem, n_begin: int = 0, n_count: Optional[int] = None, stream=None):
    n_count = prob.N - n_begin if n_count is None else n_count
    phi = torch.empty((prob.B, n_count), dtype=torch.float32, device=prob.device)
    mol_score(prob, n_begin, n_count, phi, stream)
    return phi


def topk_exact(prob: Problem, k: int, ws=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    ws = workspace(prob, MOL_OP_TOPK_EXACT, k=k) if ws is None else ws
    s = torch.empty((prob.B, k), dtype=torch.float32, device=prob.device)
    i = torch.empty((prob.B, k), dtype=torch.int32, device=prob.device)
    mol_topk_exact(prob, k, s, i, ws, stream)
    return s, i


def _topk_out(prob: Problem, k: int):
    return (torch.empty((prob.B, k), dtype=torch.float32, device=prob.device),
            torch.empty((prob.B, k), dtype=torch.int32, device=prob.device))


def topk_exact_bounded(prob: Problem, k: int, bound: torch.Tensor, ws=None, stream=None):
    """Exact top-k among items whose max component dot can reach bound[b]."""
    ws = workspace(prob, MOL_OP_TOPK_BOUNDED, k=k) if ws is None else ws
    s, i = _topk_out(prob, k)
    mol_topk_exact_bounded(prob, k, bound, s, i, ws, stream)
    return s, i


def topk_two_pass(prob: Problem, k: int, mode: int = MOL_TWO_PASS_MIN, ws=None, stream=None):
    """Algorithm 1: (scores, ids, bound used per query)."""
    ws = workspace(prob, MOL_OP_TOPK_TWO_PASS, k=k) if ws is None else ws
    s, i = _topk_out(prob, k)
    bound = torch.empty((prob.B,), dtype=torch.float32, device=prob.device)
    mol_topk_two_pass(prob, k, mode, s, i, bound, ws, stream)
    return s, i, bound


def topk_maxdot(prob: Problem, k: int, ws=None, stream=None):
    """Top-k by max_p s_p: (max dots, ids)."""
    ws = workspace(prob, MOL_OP_TOPK_MAXDOT, k=k) if ws is None else ws
    s, i = _topk_out(prob, k)
    mol_topk_maxdot(prob, k, s, i, ws, stream)
    return s, i


def topk_per_embd(prob: Problem, kprime: int, ws=None, stream=None):
    ws = workspace(prob, MOL_OP_TOPK_PER_EMBD, kprime=kprime) if ws is None else ws
    s = torch.empty((prob.B, prob.P, kprime), dtype=torch.float32, device=prob.device)
    i = torch.empty((prob.B, prob.P, kprime), dtype=torch.int32, device=prob.device)
    mol_topk_per_embd(prob, kprime, s, i, ws, stream)
    return s, i


def rerank(prob: Problem, cand: torch.Tensor, k: int, ws=None, stream=None,
           cand2: Optional[torch.Tensor] = None):
    """Union of the candidate rows of cand [B][C] (and cand2 [B][C2]),
    deduplicated and reranked with full MoL: (scores, ids, n_unique)."""
    C = cand.shape[1]
    C2 = 0 if cand2 is None else cand2.shape[1]
    ws = workspace(prob, MOL_OP_RERANK, k=k, C=C + C2) if ws is None else ws
    s = torch.empty((prob.B, k), dtype=torch.float32, device=prob.device)
    i = torch.empty((prob.B, k), dtype=torch.int32, device=prob.device)
    nu = torch.empty((prob.B,), dtype=torch.int32, device=prob.device)
    mol_rerank(prob, cand, C, cand2, C2, k, s, i, nu, ws, stream)
    return s, i, nu


def gap_bound(dots: torch.Tensor, scores: torch.Tensor, stream=None):
    """Theorem 2 certificate from per-component lists dots [B][P][m] and the
    reranked scores [B][k]: (S, S_K, bound, looser), each float32 [B]."""
    B, P, m = dots.shape
    k = scores.shape[1]
    outs = [torch.empty((B,), dtype=torch.float32, device=dots.device) for _ in range(4)]
    mol_gap_bound(B, P, m, dots, k, scores, *outs, stream=stream)
    return tuple(outs)


def gap_bound_combined(dots: torch.Tensor, ids: torch.Tensor, kprime: int, avg_ids, scores: torch.Tensor,
                       stream=None):
    """Theorem 3 certificate from per-component lists dots / ids [B][P][m]
    (m > kprime + k_avg), the TopKAvg ids [B][k_avg] (or None) and the
    reranked scores [B][k]: (S', S_K, bound), each float32 [B]."""
    B, P, m = dots.shape
    k = scores.shape[1]
    k_avg = 0 if avg_ids is None else avg_ids.shape[-1]
    outs = [torch.empty((B,), dtype=torch.float32, device=dots.device) for _ in range(3)]
    mol_gap_bound_combined(B, P, m, dots, ids, kprime, avg_ids, k_avg, k, scores, *outs, stream=stream)
    return tuple(outs)


def avg_embed(prob: Problem, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    dt = torch.bfloat16 if prob.c.dtype == MOL_BF16 else torch.float32
    q = torch.empty((prob.B, prob.d), dtype=dt, device=prob.device)
    x = torch.empty((prob.N, prob.d), dtype=dt, device=prob.device)
    mol_avg_embed(prob, q, x, stream)
    return q, x


def averaged_problem(prob: Problem, q_avg: torch.Tensor, x_avg: torch.Tensor) -> Problem:
    """The P = 1 problem TopKAvg runs on (Q = q', X = x')."""
    return Problem(q_avg.view(prob.B, 1, prob.d), x_avg.view(1, prob.N, prob.d))


# ------------------------------------------------------- learning the similarity
def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _operand(t: torch.Tensor, name: str, shape, dtypes, device) -> None:
    """Checks what the C ABI cannot see: shape (unless None), element type, device and layout."""
    if (isinstance(t, torch.Tensor) and t.dtype in dtypes and (shape is None or t.shape == shape) and
            t.device == device and t.is_contiguous()):
        return
    _need(isinstance(t, torch.Tensor), f"{name} must be a tensor")
    _need(shape is None or tuple(t.shape) == tuple(shape), f"{name} has shape {tuple(t.shape)}, needs {shape and tuple(shape)}")
    _need(t.dtype in dtypes, f"{name} has dtype {t.dtype}, needs {' or '.join(str(d) for d in dtypes)}")
    _need(t.device == device, f"{name} is on {t.device}, needs {device}")
    _need(t.is_contiguous(), f"{name} must be contiguous")


_FLOATS = (torch.float32, torch.bfloat16)
_F32_MAX = torch.finfo(torch.float32).max
_F32, _INT32 = (torch.float32,), (torch.int32,)
_HERE_NOW = contextlib.nullcontext()


def _on(device: torch.device, stream):
    """A context in which the operands' device is current, and with ``stream``
    that stream too, so that what the call allocates belongs to it."""
    if device.type != "cuda":
        raise ValueError(f"the operands are on {device}, not on a GPU")
    if stream is None and device.index == torch._C._cuda_getDevice():   # (a GPU tensor exists: no set-up to wait for)
        return _HERE_NOW
    stack = contextlib.ExitStack()
    stack.enter_context(torch.cuda.device(device))
    if stream is not None:
        s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)
        stack.enter_context(torch.cuda.stream(s))
    return stack


def _workspace(size, ws, device) -> Optional[torch.Tensor]:
    """The caller's workspace, or one of size() bytes (None for none)."""
    if ws is not None:
        if ws.dtype != torch.uint8 or ws.device != device or not ws.is_contiguous():
            raise ValueError(f"the workspace must be a contiguous uint8 tensor on {device}")
        return ws
    n = size()
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def embed_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, dtype=None, out=None, stream=None):
    """Rows of C tables by id, scaled: out[c][t] = scale table[c][ids[t]].

    table [C][V][d] float32 or bfloat16, ids int32 [T] -> [C][T][d] in
    ``dtype`` (the table's by default).  An id outside [0, V) gives a zero row.
    """
    _need(isinstance(table, torch.Tensor) and table.dim() == 3, "table must be a tensor [C][V][d]")
    _need(isinstance(ids, torch.Tensor) and ids.dim() == 1, "ids must be a tensor [T]")
    dev, (C, V, d), (T,) = table.device, table.shape, ids.shape
    dtype = (table.dtype if out is None else out.dtype) if dtype is None else dtype
    if dtype not in _FLOATS:
        raise ValueError(f"unsupported output dtype {dtype}")
    _operand(table, "table", None, _FLOATS, dev)
    _operand(ids, "ids", None, _INT32, dev)
    _sizes(C, V, d, T)
    with _on(dev, stream):
        if out is None:
            out = table.new_empty((C, T, d), dtype=dtype)
        else:
            _operand(out, "out", (C, T, d), (dtype,), dev)
        _check(load().mol_embed_lookup(table.data_ptr(), _DTYPES[table.dtype], C, V, d, ids.data_ptr(), T, scale,
                                       out.data_ptr(), _DTYPES[dtype], _stream(stream)))
    return out


def embed_grad_workspace(grad: torch.Tensor, V: int) -> torch.Tensor:
    """The workspace of embed_grad for a gradient [C][T][d] of tables of V rows."""
    C, T, d = grad.shape
    return torch.empty(max(mol_embed_grad_workspace(C, V, d, T), 1), dtype=torch.uint8, device=grad.device)


def embed_grad(grad: torch.Tensor, ids: torch.Tensor, V: int, scale: float = 1.0, dtype=torch.float32, out=None,
               accumulate: bool = False, ws=None, stream=None):
    """Gradient of embed_lookup for its tables: the rows of grad [C][T][d]
    summed by id into [C][V][d], times ``scale``.

    ``accumulate`` adds to the rows of ``out`` that have tokens and leaves the
    others as they are; otherwise every row is written.
    """
    _need(isinstance(grad, torch.Tensor) and grad.dim() == 3, "grad must be a tensor [C][T][d]")
    C, T, d = grad.shape
    dev = grad.device
    _operand(grad, "grad", None, _FLOATS, dev)
    _operand(ids, "ids", (T,), _INT32, dev)
    _sizes(C, V, d, T)
    _need(out is not None or not accumulate, "accumulate needs out")
    dtype = dtype if out is None else out.dtype
    if dtype not in _FLOATS:
        raise ValueError(f"unsupported output dtype {dtype}")
    with _on(dev, stream):
        ws = _workspace(lambda: mol_embed_grad_workspace(C, V, d, T), ws, dev)
        if out is None:
            out = grad.new_empty((C, V, d), dtype=dtype)
        else:
            _operand(out, "out", (C, V, d), (dtype,), dev)
        _check(load().mol_embed_grad(grad.data_ptr(), _DTYPES[grad.dtype], C, V, d, ids.data_ptr(), T, scale,
                                     int(accumulate), out.data_ptr(), _DTYPES[dtype], None if ws is None else ws.data_ptr(),
                                     0 if ws is None else ws.numel(), _stream(stream)))
    return out


def softmax_loss(phi: torch.Tensor, target: torch.Tensor, ids: Optional[torch.Tensor] = None, inv_temp: float = 1.0,
                 row_weight: Optional[torch.Tensor] = None, dphi: Optional[torch.Tensor] = None, ws=None, stream=None):
    """Sampled-softmax loss of score rows phi [B][N] with the positives'
    columns target int32 [B], and its gradient: (loss [B], dphi [B][N]).

    ids int32 [N]: the columns' items; a column with a negative id, or with the
    positive's id in another place than the positive's, is left out (an id past
    the tables, an empty slot to embed_lookup, is not: make it negative).  dphi is
    the gradient of sum_b row_weight[b] loss[b] (weights of 1 by default) and
    may be written over phi.
    """
    _need(isinstance(phi, torch.Tensor) and phi.dim() == 2, "phi must be a tensor [B][N]")
    B, N = phi.shape
    dev = phi.device
    _operand(phi, "phi", None, _F32, dev)
    _operand(target, "target", (B,), _INT32, dev)
    if ids is not None:
        _operand(ids, "ids", (N,), _INT32, dev)
    if row_weight is not None:
        _operand(row_weight, "row_weight", (B,), _F32, dev)
    if dphi is not None:
        _operand(dphi, "dphi", (B, N), _F32, dev)
    _sizes(B, N)
    with _on(dev, stream):
        ws = _workspace(lambda: mol_softmax_loss_workspace(B, N), ws, dev)
        loss = phi.new_empty((B,))
        if dphi is None:
            dphi = phi.new_empty((B, N))
        _check(load().mol_softmax_loss(
            B, N, phi.data_ptr(), target.data_ptr(), None if ids is None else ids.data_ptr(), inv_temp,
            None if row_weight is None else row_weight.data_ptr(), loss.data_ptr(), dphi.data_ptr(),
            None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream(stream)))
    return loss, dphi


def _check_problem(prob: Problem) -> None:
    """What the gradients rely on: every tensor of the sizes, type and device that Q, X and W1 imply."""
    B, N, P, d, H, e = prob.B, prob.N, prob.P, prob.d, prob.H, prob.tensors[0].dtype
    f32 = torch.float32
    _sizes(B, N, P, d, H)
    _need(all(t is not None for t in prob.tensors), "the problem lacks a gating tensor")
    for name, t, n, dt in zip(("Q", "X", "a_q", "a_x", "W1", "b1", "W2", "b2"), prob.tensors,
                              (B * prob.Pq * d, prob.Px * N * d, B * P, N * P, H * P, H, P * H, P),
                              (e, e, f32, f32, e, f32, e, f32)):
        _need(t.numel() == n, f"{name} has {t.numel()} elements, needs {n}")
        _need(t.dtype == dt, f"{name} has dtype {t.dtype}, needs {dt}")
        _need(t.device == prob.device, f"{name} is on {t.device}, needs {prob.device}")
    prob.checked = True


_GRADS = ("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2")


def score_grad(prob: Problem, dphi: torch.Tensor, ws=None, stream=None, only: Optional[Sequence[str]] = None,
               out: Optional[dict] = None):
    """Gradients of score(prob) for the problem's tensors, given dphi [B][N]:
    a dict of dQ, dX, da_q, da_x, dW1, db1, dW2 and db2 (or those in ``only``),
    each of its tensor's shape and type.  out: tensors to write some of them to.
    Problems with MOL_FLAG_F32_GATING: float32 throughout; bf16 ones without it keep
    16 bits of what dQ, dX, dW1 and dW2 are summed from."""
    _operand(dphi, "dphi", (prob.B, prob.N), (torch.float32,), prob.device)
    names = _GRADS if only is None else tuple(only)
    if only is not None and not all(n in _GRADS for n in names):
        raise ValueError(f"unknown gradient in {names}: {', '.join(_GRADS)}")
    if not prob.checked:
        _check_problem(prob)
    if out is not None and not set(out) <= set(names):
        raise ValueError(f"out holds {sorted(out)}, gradients are {', '.join(names)}")
    with _on(prob.device, stream):
        ws = _workspace(lambda: mol_workspace_size(prob, MOL_OP_SCORE_GRAD), ws, prob.device)
        got, c = {}, MolScoreGradsC()
        for g, t in zip(_GRADS, prob.tensors):
            if g not in names:
                continue
            if out is not None and g in out:
                _operand(out[g], g, t.shape, (t.dtype,), prob.device)
                got[g] = out[g]
            else:
                got[g] = torch.empty_like(t)
            setattr(c, g, got[g].data_ptr())
        _check(load().mol_score_grad(prob.ref, dphi.data_ptr(), ctypes.byref(c), None if ws is None else ws.data_ptr(),
                                     0 if ws is None else ws.numel(), _stream(stream)))
    return got


class AdamwTensors:
    """The tensors of an AdamW step and their states, laid out once for the
    library (and kept alive by this object).

    p, g: lists of float32 or bfloat16 tensors; m, v: float32, or 8-bit
    (float8_e4m3fn codes, with m_scale and v_scale float32 [ceil(n / 256)]).
    weight_decay: one number, or one a tensor.  out: None (in place), or a
    dict of lists "p", "m", "v" (and "m_scale", "v_scale") to write the new
    state to, and "copy": bfloat16 copies of the new parameters, whole or for
    some tensors (None for the others); any may be missing or None.  Tensors
    keep their place in the stream of random numbers that rounds 8-bit states
    by their order: each starts at a multiple of 256.

    Making a plan takes about 11 us a tensor on the host (24 tensors: 270 us,
    their step 17), so that it is for tensors that stay where they are.
    """

    def __init__(self, p: List[torch.Tensor], g: List[torch.Tensor], m: List[torch.Tensor], v: List[torch.Tensor],
                 m_scale: Optional[List[torch.Tensor]] = None, v_scale: Optional[List[torch.Tensor]] = None,
                 weight_decay=0.0, out: Optional[dict] = None):
        # (lists of its own: the descriptors hold addresses, which the caller's lists may let go of)
        p, g, m, v = tuple(p), tuple(g), tuple(m), tuple(v)
        m_scale, v_scale = (None if x is None else tuple(x) for x in (m_scale, v_scale))
        out = {k: tuple(x) for k, x in (out or {}).items() if x is not None}
        n = len(p)
        lists = {"g": g, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale}
        unknown = set(out) - {"p", "m", "v", "m_scale", "v_scale", "copy"}
        _need(not unknown, f"unknown outputs {sorted(unknown)}")
        for name, x in list(lists.items()) + list(out.items()):
            _need(x is None or len(x) == n, f"{name} has not the {n} entries of p")
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        _need(len(decay) == n, f"weight_decay has not the {n} entries of p")
        _need(all(isinstance(t, torch.Tensor) for t in p), "p must hold tensors")
        self.n, self.device = n, p[0].device if n else torch.device("cuda")
        self.c = (MolAdamwTensorC * max(n, 1))()
        self.tensors = (p, g, m, v, m_scale, v_scale, out)
        dev, index = self.device, p[0].get_device() if n else 0

        def at(t, name, i, shape, dtypes):             # (a plan of many tensors is made of thousands of these checks)
            if not (isinstance(t, torch.Tensor) and t.dtype in dtypes and t.shape == shape and t.get_device() == index and
                    t.is_contiguous()):
                _operand(t, f"{name}[{i}]", shape, dtypes, dev)
            return t.data_ptr()

        def new(name, i, shape, dtypes, old):          # where an output goes: in place unless out has it
            return at(out[name][i], "out " + name, i, shape, dtypes) if name in out else old

        f32, e4m3, bf16, copies = (torch.float32,), (torch.float8_e4m3fn,), (torch.bfloat16,), out.get("copy")
        offset = 0
        for i, t in enumerate(p):
            shape, count = t.shape, t.numel()
            blocks = (count + MOL_STATE_BLOCK - 1) // MOL_STATE_BLOCK
            eight = isinstance(m[i], torch.Tensor) and m[i].dtype == torch.float8_e4m3fn
            state = e4m3 if eight else f32
            pp, gp = at(t, "p", i, shape, _FLOATS), at(g[i], "g", i, shape, _FLOATS)
            mp, vp = at(m[i], "m", i, shape, state), at(v[i], "v", i, shape, state)
            ms = vs = mso = vso = None
            if eight:
                _need(m_scale is not None and v_scale is not None, "8-bit states need m_scale and v_scale")
                _need(("m" in out) == ("m_scale" in out) and ("v" in out) == ("v_scale" in out),
                      "outputs m and m_scale, v and v_scale go together")
                ms, vs = at(m_scale[i], "m_scale", i, (blocks,), f32), at(v_scale[i], "v_scale", i, (blocks,), f32)
                mso, vso = new("m_scale", i, (blocks,), f32, ms), new("v_scale", i, (blocks,), f32, vs)
            self.c[i] = MolAdamwTensorC(
                count, pp, gp, mp, vp, ms, vs, new("p", i, shape, (t.dtype,), pp), new("m", i, shape, state, mp),
                new("v", i, shape, state, vp), mso, vso,
                None if copies is None or copies[i] is None else at(copies[i], "out copy", i, shape, bf16),
                _DTYPES[t.dtype], _DTYPES[g[i].dtype], MOL_STATE_E4M3 if eight else MOL_STATE_F32, decay[i], offset)
            offset += blocks * MOL_STATE_BLOCK


def adamw_step(tensors: AdamwTensors, lr=1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, step=1,
               seed: int = 0, grad_scale: Optional[torch.Tensor] = None, stream=None) -> None:
    """One AdamW step over all of ``tensors``.

    lr and step (from 1) are numbers, or one-element tensors on the GPU
    (float32, int32) that the kernel reads, for graphs that are replayed;
    grad_scale: None, or one float32 on the GPU that multiplies every gradient.
    """
    if tensors.n == 0:
        return
    for name, t, dt in (("lr", lr, torch.float32), ("step", step, torch.int32), ("grad_scale", grad_scale, torch.float32)):
        if isinstance(t, torch.Tensor):
            _need(t.numel() == 1, f"{name} must have one element")
            _operand(t, name, t.shape, (dt,), tensors.device)
        else:
            _need(name != "grad_scale" or t is None, "grad_scale must be a tensor")
    on_lr, on_step = isinstance(lr, torch.Tensor), isinstance(step, torch.Tensor)
    if not on_step and step >= 1 << 31:
        raise ValueError(f"step = {step} is not below 2^31")
    opt = MolAdamwC(0.0 if on_lr else lr, beta1, beta2, eps, 1 if on_step else step, seed & 0xFFFFFFFF, _ptr(grad_scale),
                    _ptr(lr) if on_lr else None, _ptr(step) if on_step else None)
    with _on(tensors.device, stream):
        mol_adamw_step(opt, tensors.c, tensors.n, stream)


class Learner:
    """One model in training by the sampled-softmax objective: embedding tables
    and gating parameters, their bfloat16 copies that the kernels score with,
    gradients and AdamW states, all laid out once.

    queries [Vq][Pq][d] and items [Px][V][d]: the component embeddings' float32
    masters; a_q [Vq][P], a_x [V][P]: the gating logits of every query and item;
    W1 [H][P], b1 [H], W2 [P][H], b2 [P]: the gating MLP, all float32 (they are
    updated in place).  weight_decay is for the embeddings and W1, W2.  The rows
    are learned and served as they are: Eq. 2's L2 normalisation of the components is
    not part of a step, so that it is a model of unnormalised dot products.
    states_8bit: AdamW states of the two embedding tables in 8 bits.  flags: the
    precision of the gating MLP in a step's scores (MOL_FLAG_*); float32 by default,
    since training moves its weights out of the range that the others are meant for
    (1024 x 2048 pairs of 8 x 8: 430 us of a step's 1580; 0 takes 90, with weights of RMS
    up to 0.3, MOL_FLAG_BF16X2_GATING 130, up to 1).  grad_flags: the same for the
    gradients, whose chain has no such range; MOL_FLAG_F32_GATING keeps float32 up to
    their rounding to bf16 (see score_grad).

    The copy of the items' table is laid out as a corpus: ``problem`` gives the
    retrieval problem of the model as it is.

    To save a learner: ``master``, ``state`` (m and v, and of 8-bit states
    m_scale and v_scale, by tensor) and ``steps``.  One made of the saved masters with
    the same options, whose state and steps the saved ones are copied into, goes on bit for bit.
    """

    def __init__(self, queries, items, a_q, a_x, W1, b1, W2, b2, weight_decay: float = 0.0, states_8bit: bool = False,
                 seed: int = 0, flags: int = MOL_FLAG_F32_GATING, grad_flags: int = 0):
        Vq, Pq, d = queries.shape
        Px, V, _ = items.shape
        P, dev = Pq * Px, queries.device
        H = W1.shape[0]
        for name, t, shape in (("items", items, (Px, V, d)), ("a_q", a_q, (Vq, P)), ("a_x", a_x, (V, P)), ("W1", W1, (H, P)),
                               ("b1", b1, (H,)), ("W2", W2, (P, H)), ("b2", b2, (P,)), ("queries", queries, (Vq, Pq, d))):
            _operand(t, name, shape, (torch.float32,), dev)
        self.master = dict(queries=queries, items=items, a_q=a_q, a_x=a_x, W1=W1, b1=b1, W2=W2, b2=b2)
        self.copy = {n: self.master[n].bfloat16() for n in ("queries", "items", "W1", "W2")}
        self.grad = {n: torch.empty_like(t, dtype=torch.bfloat16 if n in ("W1", "W2") else torch.float32)
                     for n, t in self.master.items()}
        eight = {n: states_8bit and n in ("queries", "items") for n in self.master}
        state = lambda n, t: torch.zeros_like(t, dtype=torch.float8_e4m3fn if eight[n] else torch.float32)  # noqa: E731
        scale = lambda n, t: (torch.zeros((t.numel() + MOL_STATE_BLOCK - 1) // MOL_STATE_BLOCK, device=dev)  # noqa: E731
                              if eight[n] else None)
        m, v = ({n: state(n, t) for n, t in self.master.items()} for _ in range(2))
        ms, vs = ([scale(n, t) for n, t in self.master.items()] for _ in range(2))
        self.tensors = AdamwTensors(
            list(self.master.values()), list(self.grad.values()), list(m.values()), list(v.values()), ms, vs,
            weight_decay=[weight_decay if n in self.copy else 0.0 for n in self.master],
            out=dict(copy=[self.copy.get(n) for n in self.master]))
        self.state = dict(m=m, v=v)
        if any(eight.values()):
            for k, x in (("m_scale", ms), ("v_scale", vs)):
                self.state[k] = {n: t for n, t in zip(self.master, x) if t is not None}
        self.steps = torch.zeros(1, dtype=torch.int32, device=dev)   # on the GPU, so that a captured step counts on
        self.seed, self.flags, self.grad_flags = seed, flags, grad_flags
        self.shape = (Vq, V, Pq, Px, P, d)

    def step(self, query_ids: torch.Tensor, item_ids: torch.Tensor, target: torch.Tensor, lr,
             inv_temp: float = 20.0) -> torch.Tensor:
        """One optimisation step on B queries and N sampled items: query_ids int32
        [B] (outside the table: a row of zeros, which adds to no gradient), item_ids
        int32 [N] (outside the table: an empty slot, no candidate), target int32 [B]:
        the column of each query's positive; lr: a number, or one float32 on the GPU
        (which a captured step reads when it runs).  Returns the losses [B] from
        before the step.  Allocates with torch and launches on the current stream
        only: it can be captured into a graph."""
        # (what AdamW and the loss would refuse, before anything is changed)
        if isinstance(lr, torch.Tensor):
            _need(lr.numel() == 1, "lr must have one element")
            _operand(lr, "lr", lr.shape, (torch.float32,), self.steps.device)
        elif not isinstance(lr, numbers.Real) or not 0 <= lr <= _F32_MAX:
            raise ValueError(f"lr = {lr!r} is not a rate: a number from 0 to {_F32_MAX:g}")
        _need(query_ids.numel() > 0 and item_ids.numel() > 0, "a step needs a query and an item")
        with _on(self.steps.device, None):
            return self._step(query_ids, item_ids, target, lr, inv_temp)

    def _step(self, query_ids, item_ids, target, lr, inv_temp) -> torch.Tensor:
        Vq, V, Pq, Px, P, d = self.shape
        B, N = query_ids.numel(), item_ids.numel()
        M, C, G = self.master, self.copy, self.grad
        queries = C["queries"].view(1, Vq, Pq * d)
        item_ids = item_ids.masked_fill(item_ids >= V, -1)       # (the loss takes negative ids alone for empty slots)
        tensors = (embed_lookup(queries, query_ids).view(B, Pq, d), embed_lookup(C["items"], item_ids),
                   embed_lookup(M["a_q"].view(1, Vq, P), query_ids).view(B, P),
                   embed_lookup(M["a_x"].view(1, V, P), item_ids).view(N, P), C["W1"], M["b1"], C["W2"], M["b2"])
        phi = score(Problem(*tensors, flags=self.flags))
        weight = torch.full((B,), 1.0 / B, device=phi.device)
        loss, dphi = softmax_loss(phi, target, item_ids, inv_temp, weight, dphi=phi)
        g = score_grad(Problem(*tensors, flags=self.grad_flags), dphi, out=dict(dW1=G["W1"], db1=G["b1"], dW2=G["W2"], db2=G["b2"]))
        embed_grad(g["dQ"].view(1, B, Pq * d), query_ids, Vq, out=G["queries"].view(1, Vq, Pq * d))
        embed_grad(g["dX"], item_ids, V, out=G["items"])
        embed_grad(g["da_q"].view(1, B, P), query_ids, Vq, out=G["a_q"].view(1, Vq, P))
        embed_grad(g["da_x"].view(1, N, P), item_ids, V, out=G["a_x"].view(1, V, P))
        self.steps.add_(1)
        adamw_step(self.tensors, lr=lr, step=self.steps, seed=self.seed)
        return loss

    def problem(self, query_ids: torch.Tensor, flags: int = 0) -> Problem:
        """The retrieval problem of these queries against all items.  flags: 0 is
        meant for gating weights of RMS up to 0.3 (see MOL_FLAG_*)."""
        Vq, V, Pq, Px, P, d = self.shape
        B = query_ids.numel()
        return Problem(embed_lookup(self.copy["queries"].view(1, Vq, Pq * d), query_ids).view(B, Pq, d), self.copy["items"],
                       embed_lookup(self.master["a_q"].view(1, Vq, P), query_ids).view(B, P), self.master["a_x"],
                       self.copy["W1"], self.master["b1"], self.copy["W2"], self.master["b2"], flags)
