"""ctypes binding of libla (include/la.h): argument marshalling only.

Every step of selection and attention runs in the HIP kernels of libla.so; this
module checks tensor shapes, dtypes and devices, allocates outputs and the
workspace with torch, and passes raw device pointers and torch's current HIP
stream across the C ABI.  There is no fallback: a missing library or a non-GPU
tensor raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libla.so")

LA_OK, LA_ERR_ARG, LA_ERR_SHAPE, LA_ERR_WORKSPACE, LA_ERR_HIP = range(5)


class Shape(ctypes.Structure):
    """la_shape."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "Lq", "Lk", "d", "block", "n_text", "frame_tokens")]

    def __repr__(self):
        return "Shape(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class LaError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {status_string(status)} (status {status})")
        self.status = status


class Grid3D(ctypes.Structure):
    """la_grid3d: 3-D block layout of one AR chunk (text, context frames, chunk frames)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "d", "n_text", "T_ctx", "T_q", "Hs", "Ws", "bt", "bh", "bw",
                                              "block")]

    def __repr__(self):
        return "Grid3D(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class RopeShape(ctypes.Structure):
    """la_rope_shape."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "Hq", "Hk", "d", "rot", "interleaved", "dtype", "axes")] + \
               [("section", ctypes.c_int32 * 3)] + \
               [(f"{t}_{n}", ctypes.c_int64) for t in ("q", "qo", "k", "ko") for n in ("batch", "token", "head")]


class Seqs(ctypes.Structure):
    """la_seqs: packed sequences and the strides of their tensors."""
    _fields_ = [(n, ctypes.c_int32) for n in ("S", "Tq", "Tk", "Hq", "Hkv", "d", "causal")] + \
               [(n, ctypes.c_int64) for n in ("q_token", "q_head", "o_token", "o_head", "k_token", "k_head", "v_token",
                                              "v_head")]


class Kv4(ctypes.Structure):
    """la_kv4: the pages of a 4-bit cache."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page", "max_pages")]


LA_PART_TEXT, LA_PART_CONTEXT, LA_PART_CHUNK, LA_PART_ALL = 1, 2, 4, 7

_lib = None
_fns = {}          # the functions of _lib by name
_P = ctypes.c_void_p
_SP = ctypes.POINTER(Shape)
_GP = ctypes.POINTER(Grid3D)
_QP = ctypes.POINTER(Seqs)
_KP = ctypes.POINTER(Kv4)
_RP = ctypes.POINTER(RopeShape)

_SIGNATURES = {
    "la_workspace_bytes": (ctypes.c_size_t, [_SP]),
    "la_select_blocks": (ctypes.c_int, [_SP, _P, _P, ctypes.c_float, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_select_blocks_topk": (ctypes.c_int, [_SP, _P, _P, ctypes.c_int32, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_select_blocks_noalloc": (ctypes.c_int, [_SP, _P, _P, ctypes.c_float, _P, _P, _P, _P]),
    "la_sparse_attn_fwd": (ctypes.c_int, [_SP, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_sparse_attn_plan": (ctypes.c_int, [_SP, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_sparse_attn_run": (ctypes.c_int, [_SP, _P, _P, _P, ctypes.c_float, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_sparse_attn_merge": (ctypes.c_int, [_SP, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_sparse_attn_schedule": (ctypes.c_int, [_SP, _P, ctypes.c_size_t, _P, _P, _P, _P, _P, _P, _P]),
    "la_mask_to_list": (ctypes.c_int, [_SP, _P, _P, _P, _P]),
    "la_grid3d_shape": (ctypes.c_int, [_GP, _SP]),
    "la_grid3d_valid": (ctypes.c_int, [_GP, _P, _P]),
    "la_prep_q_3d": (ctypes.c_int, [_GP, _P, _P, _P, _P]),
    "la_prep_kv_3d": (ctypes.c_int, [_GP, _P, _P, ctypes.c_uint32, _P, _P, _P, _P]),
    "la_pool_blocks": (ctypes.c_int, [_SP, _P, ctypes.c_int32, _P, _P]),
    "la_select_pooled": (ctypes.c_int, [_SP, _P, _P, ctypes.c_float, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_select_pooled_topk": (ctypes.c_int, [_SP, _P, _P, ctypes.c_int32, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_sparse_attn_fwd_valid": (ctypes.c_int, [_SP, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P,
                                                ctypes.c_size_t, _P]),
    "la_sparse_attn_plan_valid": (ctypes.c_int, [_SP, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_untile_o_3d": (ctypes.c_int, [_GP, _P, _P, _P, _P, _P]),
    "la_rope": (ctypes.c_int, [_RP, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P]),
    "la_prompt_ws_bytes": (ctypes.c_size_t, [_QP]),
    "la_prompt_attn": (ctypes.c_int, [_QP, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, ctypes.c_size_t, _P]),
    "la_kv4_page_bytes": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32]),
    "la_kv4_append": (ctypes.c_int, [_QP, _KP, _P, _P, _P, _P, _P, _P, _P]),
    "la_kv4_read": (ctypes.c_int, [_QP, _KP, _P, _P, _P, _P, _P, _P, _P]),
    "la_kv4_ws_bytes": (ctypes.c_size_t, [_QP, _KP, ctypes.c_int32]),
    "la_kv4_attn": (ctypes.c_int, [_QP, _KP, ctypes.c_int32, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P,
                                   ctypes.c_size_t, _P]),
    "la_latent_mse": (ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int32, _P, _P, ctypes.c_size_t, _P]),
    "la_dynamics_ema": (ctypes.c_int, [ctypes.c_double, _P, ctypes.c_double, _P]),
    "la_temporal_window": (ctypes.c_int, [ctypes.c_double, ctypes.c_double, ctypes.c_int32, _P]),
    "la_pose_revisiting": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_float, _P]),
    "la_denoise_schedule": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, _P]),
    "la_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "la_abi_version": (ctypes.c_int32, []),
}


def lib() -> ctypes.CDLL:
    """Loads libla.so (torch first, so the library binds to the HIP runtime torch loaded)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(or python -m paper_2605_31158_amd.build)")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
            _fns[name] = fn
        _lib = h
    return _lib


def status_string(status: int) -> str:
    return lib().la_status_string(status).decode()


def make_shape(B, H, Lq, Lk, d, block, n_text=0, frame_tokens=0) -> Shape:
    return Shape(B, H, Lq, Lk, d, block, n_text, frame_tokens)


def workspace_bytes(shape: Shape) -> int:
    return int(lib().la_workspace_bytes(ctypes.byref(shape)))


# Small calls are bound by the host: arguments go to ctypes as plain numbers (the signatures convert
# them), and the stream's handle is asked for directly; a torch.cuda.Stream object for it costs 2.1 us
# of the 10.5 a latent_mse call took, the handle 0.1.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(t: torch.Tensor):
    if _raw_stream is not None and t.is_cuda:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _check_qkv(name, t: torch.Tensor, B=None, H=None, d=None):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != torch.bfloat16 or t.dim() != 4 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous bfloat16 [B, H, L, d] tensor")
    if (B is not None and t.shape[0] != B) or (H is not None and t.shape[1] != H) or \
            (d is not None and t.shape[3] != d):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, inconsistent with the other operands")


def _workspace(shape: Shape, device, ws: Optional[torch.Tensor]):
    need = workspace_bytes(shape)
    if need == 0 and ws is None:
        return None, 0
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return ws, ws.numel()


def _call(fn: str, *args):
    if _lib is None:
        lib()
    st = _fns[fn](*args)
    if st != LA_OK:
        raise LaError(fn, st)


def nblocks(L: int, block: int) -> int:
    return -(-L // block)


def select_blocks(q: torch.Tensor, k: torch.Tensor, block: int, tau: float, n_text: int = 0,
                  want_mask: bool = True, ws: Optional[torch.Tensor] = None,
                  out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None):
    """Cumulative-mass block selection -> (mask uint8 [B,H,NQ,NK] or None, counts int32 [B,H,NQ],
    idx int32 [B,H,NQ,NK] ascending in the first counts[] slots)."""
    return _select("la_select_blocks", ctypes.c_float(tau), q, k, block, n_text, want_mask, ws, out)


def select_blocks_topk(q: torch.Tensor, k: torch.Tensor, block: int, keep_blocks: int, n_text: int = 0,
                       want_mask: bool = True, ws: Optional[torch.Tensor] = None,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None):
    """Top-keep_blocks selection (the paper's Top-floor(rM) rule with keep_blocks = floor(r*M))."""
    return _select("la_select_blocks_topk", ctypes.c_int32(keep_blocks), q, k, block, n_text, want_mask, ws, out)


def select_blocks_noalloc(q: torch.Tensor, k: torch.Tensor, block: int, tau: float, mask: Optional[torch.Tensor],
                          counts: torch.Tensor, idx: torch.Tensor, n_text: int = 0):
    """la_select_blocks_noalloc into the caller's outputs (mask may be None): the library's own
    scratch instead of a workspace, nothing allocated by the call or here."""
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    _check_qkv("k", k, B, H, d)
    shape = make_shape(B, H, Lq, k.shape[2], d, block, n_text, 0)
    _call("la_select_blocks_noalloc", ctypes.byref(shape), _ptr(q), _ptr(k), ctypes.c_float(tau), _ptr(mask),
          _ptr(counts), _ptr(idx), _stream(q))


def _select(fn, rule_arg, q, k, block, n_text, want_mask, ws, out):
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    _check_qkv("k", k, B, H, d)
    Lk = k.shape[2]
    shape = make_shape(B, H, Lq, Lk, d, block, n_text, 0)
    NQ, NK = nblocks(Lq, block), nblocks(Lk, block)
    if out is None:
        mask = torch.empty((B, H, NQ, NK), dtype=torch.uint8, device=q.device) if want_mask else None
        counts = torch.empty((B, H, NQ), dtype=torch.int32, device=q.device)
        idx = torch.empty((B, H, NQ, NK), dtype=torch.int32, device=q.device)
    else:
        mask, counts, idx = out
    ws, nbytes = _workspace(shape, q.device, ws)
    _call(fn, ctypes.byref(shape), _ptr(q), _ptr(k), rule_arg, _ptr(mask), _ptr(counts), _ptr(idx),
          _ptr(ws), ctypes.c_size_t(nbytes), _stream(q))
    return mask, counts, idx


def sparse_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, counts: torch.Tensor,
                    idx: torch.Tensor, block: int, scale: Optional[float] = None, n_text: int = 0,
                    frame_tokens: int = 0, want_lse: bool = False, ws: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                    kvalid: Optional[torch.Tensor] = None):
    """Block-sparse attention over the kept lists -> o bf16 [B,H,Lq,d] (and lse fp32 [B,H,Lq]).
    kvalid (int32 [NK] on the GPU): valid keys at the front of each key block
    (la_sparse_attn_fwd_valid); the other slots are padding."""
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    _check_qkv("k", k, B, H, d)
    _check_qkv("v", v, B, H, d)
    Lk = k.shape[2]
    if v.shape[2] != Lk:
        raise ValueError("k and v must have the same length")
    NQ, NK = nblocks(Lq, block), nblocks(Lk, block)
    if counts.dtype != torch.int32 or tuple(counts.shape) != (B, H, NQ) or not counts.is_contiguous():
        raise ValueError(f"counts must be contiguous int32 {(B, H, NQ)}")
    if idx.dtype != torch.int32 or tuple(idx.shape) != (B, H, NQ, NK) or not idx.is_contiguous():
        raise ValueError(f"idx must be contiguous int32 {(B, H, NQ, NK)}")
    shape = make_shape(B, H, Lq, Lk, d, block, n_text, frame_tokens)
    o = out if out is not None else torch.empty_like(q)
    lse = lse_out if lse_out is not None else (
        torch.empty((B, H, Lq), dtype=torch.float32, device=q.device) if want_lse else None)
    ws, nbytes = _workspace(shape, q.device, ws)
    sc = ctypes.c_float(scale if scale is not None else 0.0)
    if kvalid is None:
        _call("la_sparse_attn_fwd", ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(counts), _ptr(idx), sc,
              _ptr(o), _ptr(lse), _ptr(ws), ctypes.c_size_t(nbytes), _stream(q))
    else:
        if kvalid.device != q.device or kvalid.dtype != torch.int32 or tuple(kvalid.shape) != (NK,):
            raise ValueError(f"kvalid must be an int32 [{NK}] tensor on {q.device}")
        _call("la_sparse_attn_fwd_valid", ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(counts), _ptr(idx),
              _ptr(kvalid), sc, _ptr(o), _ptr(lse), _ptr(ws), ctypes.c_size_t(nbytes), _stream(q))
    return (o, lse) if (want_lse or lse_out is not None) else o


class BoundCall:
    """One C-ABI call with its arguments marshalled once (tensors, shape, stream fixed), for
    loops that issue the same call many times; calling it returns nothing and raises LaError
    on a failed status."""

    def __init__(self, fn: str, *args, keep=()):
        self._name = fn
        self._fn = getattr(lib(), fn)
        self._args = args
        self._keep = keep          # tensors and structs the raw pointers refer to

    def __call__(self):
        st = self._fn(*self._args)
        if st != LA_OK:
            raise LaError(self._name, st)


LA_POOL_Q, LA_POOL_K = 0, 1


def pool_blocks(x: torch.Tensor, block: int, which: str, shape: Shape, out: Optional[torch.Tensor] = None):
    """Block means of q (which="q", -> [B,H,NQ,d]) or k (which="k", -> [B,H,NK,d]) of `shape`, fp32;
    a ragged last block is the mean of its valid rows."""
    wcode = {"q": LA_POOL_Q, "k": LA_POOL_K}[which]
    L = shape.Lq if which == "q" else shape.Lk
    _check_qkv(which, x, shape.B, shape.H, shape.d)
    if x.shape[2] != L:
        raise ValueError(f"{which} must hold {L} tokens")
    nb = nblocks(L, block)
    if out is None:
        out = torch.empty((shape.B, shape.H, nb, shape.d), dtype=torch.float32, device=x.device)
    _call("la_pool_blocks", ctypes.byref(shape), _ptr(x), ctypes.c_int32(wcode), _ptr(out), _stream(x))
    return out


def bind_attn_steps(q, k, v, counts, idx, block, o, ws, scale: Optional[float] = None, n_text: int = 0,
                    frame_tokens: int = 0, lse: Optional[torch.Tensor] = None):
    """(plan, run, merge) of la_sparse_attn_fwd as BoundCalls on fixed tensors and the current
    stream; plan + run + merge computes the same o (and lse) as sparse_attn_fwd.  One plan serves
    any number of runs, as long as no other call uses `ws` in between (a selection call writes
    its scores there): after such a call, plan again before the next run."""
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    _check_qkv("k", k, B, H, d)
    _check_qkv("v", v, B, H, d)
    Lk = k.shape[2]
    shape = make_shape(B, H, Lq, Lk, d, block, n_text, frame_tokens)
    nbytes = ctypes.c_size_t(ws.numel())
    st = _stream(q)
    keep = (q, k, v, counts, idx, o, ws, lse, shape)
    sc = ctypes.c_float(scale if scale is not None else 0.0)
    plan = BoundCall("la_sparse_attn_plan", ctypes.byref(shape), _ptr(counts), _ptr(idx), _ptr(ws), nbytes, st,
                     keep=keep)
    run = BoundCall("la_sparse_attn_run", ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), sc, _ptr(o), _ptr(lse),
                    _ptr(ws), nbytes, st, keep=keep)
    merge = BoundCall("la_sparse_attn_merge", ctypes.byref(shape), _ptr(o), _ptr(lse), _ptr(ws), nbytes, st,
                      keep=keep)
    return plan, run, merge


def plan_schedule(shape: Shape, ws: torch.Tensor) -> dict:
    """The schedule of the plan in ws (la_sparse_attn_schedule): P, U and the arrays tstart
    [U+1], ucount [U], dp_start [P+1], sk_start [P+1] as int64 CPU tensors (synchronises)."""
    P, U = ctypes.c_int32(0), ctypes.c_int32(0)
    _call("la_sparse_attn_schedule", ctypes.byref(shape), _ptr(ws), ctypes.c_size_t(ws.numel()), ctypes.byref(P),
          ctypes.byref(U), None, None, None, None, _stream(ws))
    arrs = {"tstart": int(U.value) + 1, "ucount": int(U.value), "dp_start": int(P.value) + 1,
            "sk_start": int(P.value) + 1}
    bufs = {k: torch.empty(n, dtype=torch.int32, device=ws.device) for k, n in arrs.items()}
    _call("la_sparse_attn_schedule", ctypes.byref(shape), _ptr(ws), ctypes.c_size_t(ws.numel()), ctypes.byref(P),
          ctypes.byref(U), _ptr(bufs["tstart"]), _ptr(bufs["ucount"]), _ptr(bufs["dp_start"]),
          _ptr(bufs["sk_start"]), _stream(ws))
    out = {k: b.cpu().to(torch.int64) for k, b in bufs.items()}
    out["P"], out["U"] = int(P.value), int(U.value)
    return out


def bind_select_cached(q, block, tau, kbar, qbar, mask, counts, idx, ws, Lk: int, n_text: int = 0):
    """(pool Q, select from pooled means) as BoundCalls: the selection of a step whose key means
    kbar [B,H,NK,d] were pooled earlier (la_pool_blocks); qbar [B,H,NQ,d] is written."""
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    shape = make_shape(B, H, Lq, Lk, d, block, n_text, 0)
    st = _stream(q)
    keep = (q, kbar, qbar, mask, counts, idx, ws, shape)
    pool = BoundCall("la_pool_blocks", ctypes.byref(shape), _ptr(q), ctypes.c_int32(LA_POOL_Q), _ptr(qbar), st,
                     keep=keep)
    sel = BoundCall("la_select_pooled", ctypes.byref(shape), _ptr(qbar), _ptr(kbar), ctypes.c_float(tau), _ptr(mask),
                    _ptr(counts), _ptr(idx), _ptr(ws), ctypes.c_size_t(ws.numel()), st, keep=keep)
    return pool, sel


def bind_select(q, k, block, tau, mask, counts, idx, ws, n_text: int = 0) -> BoundCall:
    """la_select_blocks as a BoundCall on fixed tensors and the current stream."""
    _check_qkv("q", q)
    B, H, Lq, d = q.shape
    _check_qkv("k", k, B, H, d)
    shape = make_shape(B, H, Lq, k.shape[2], d, block, n_text, 0)
    return BoundCall("la_select_blocks", ctypes.byref(shape), _ptr(q), _ptr(k), ctypes.c_float(tau), _ptr(mask),
                     _ptr(counts), _ptr(idx), _ptr(ws), ctypes.c_size_t(ws.numel()), _stream(q),
                     keep=(q, k, mask, counts, idx, ws, shape))


def mask_to_list(mask: torch.Tensor, block: int, Lq: int, Lk: int, d: int = 128):
    """Block mask uint8 [B,H,NQ,NK] -> (counts, idx) as la_sparse_attn_fwd reads them."""
    if mask.device.type != "cuda" or mask.dtype != torch.uint8 or mask.dim() != 4 or not mask.is_contiguous():
        raise TypeError("mask must be a contiguous uint8 [B, H, NQ, NK] GPU tensor")
    B, H, NQ, NK = mask.shape
    if NQ != nblocks(Lq, block) or NK != nblocks(Lk, block):
        raise ValueError("mask shape does not match Lq, Lk and block")
    shape = make_shape(B, H, Lq, Lk, d, block, 0, 0)
    counts = torch.empty((B, H, NQ), dtype=torch.int32, device=mask.device)
    idx = torch.empty((B, H, NQ, NK), dtype=torch.int32, device=mask.device)
    _call("la_mask_to_list", ctypes.byref(shape), _ptr(mask), _ptr(counts), _ptr(idx), _stream(mask))
    return counts, idx


# ----------------------------------------------------------------------------------------------
# 3-D block layout

def grid3d(B, H, d, n_text, T_ctx, T_q, Hs, Ws, bt, bh, bw, block=128) -> Grid3D:
    return Grid3D(B, H, d, n_text, T_ctx, T_q, Hs, Ws, bt, bh, bw, block)


def grid3d_shape(g: Grid3D) -> Shape:
    """la_shape of the tiled problem (Lq = NQ block, Lk = NK block, n_text = NT block)."""
    shape = Shape()
    _call("la_grid3d_shape", ctypes.byref(g), ctypes.byref(shape))
    return shape


def grid3d_valid(g: Grid3D):
    """(qvalid int32 [NQ], kvalid int32 [NK]) as numpy arrays: valid tokens per block."""
    import numpy as np
    shape = grid3d_shape(g)
    qv = np.zeros(nblocks(shape.Lq, g.block), dtype=np.int32)
    kv = np.zeros(nblocks(shape.Lk, g.block), dtype=np.int32)
    _call("la_grid3d_valid", ctypes.byref(g), qv.ctypes.data_as(_P), kv.ctypes.data_as(_P))
    return qv, kv


def _check_lin(name, t, g: Grid3D, L):
    _check_qkv(name, t, g.B, g.H, g.d)
    if t.shape[2] != L:
        raise ValueError(f"{name} must hold {L} tokens, got {t.shape[2]}")


def prep_q_3d(g: Grid3D, q: torch.Tensor, q_tiled: Optional[torch.Tensor] = None,
              qbar: Optional[torch.Tensor] = None, want_qbar: bool = True):
    """Fused Q-Prep: q linear [B,H,T_q Hs Ws,d] -> (q_tiled bf16 [B,H,NQ block,d], qbar fp32 [B,H,NQ,d])."""
    _check_lin("q", q, g, g.T_q * g.Hs * g.Ws)
    shape = grid3d_shape(g)
    NQ = nblocks(shape.Lq, g.block)
    if q_tiled is None:
        q_tiled = torch.empty((g.B, g.H, shape.Lq, g.d), dtype=torch.bfloat16, device=q.device)
    if qbar is None and want_qbar:
        qbar = torch.empty((g.B, g.H, NQ, g.d), dtype=torch.float32, device=q.device)
    _call("la_prep_q_3d", ctypes.byref(g), _ptr(q), _ptr(q_tiled), _ptr(qbar), _stream(q))
    return q_tiled, qbar


def prep_kv_3d(g: Grid3D, k: torch.Tensor, v: torch.Tensor, parts: int = LA_PART_ALL,
               k_tiled: Optional[torch.Tensor] = None, v_tiled: Optional[torch.Tensor] = None,
               kbar: Optional[torch.Tensor] = None, want_kbar: bool = True):
    """Fused KV-Prep of the regions in `parts`: k, v linear [B,H,n_text+(T_ctx+T_q) Hs Ws,d] ->
    (k_tiled, v_tiled bf16 [B,H,NK block,d], kbar fp32 [B,H,NK,d])."""
    L = g.n_text + (g.T_ctx + g.T_q) * g.Hs * g.Ws
    _check_lin("k", k, g, L)
    _check_lin("v", v, g, L)
    shape = grid3d_shape(g)
    NK = nblocks(shape.Lk, g.block)
    if k_tiled is None:
        k_tiled = torch.empty((g.B, g.H, shape.Lk, g.d), dtype=torch.bfloat16, device=k.device)
    if v_tiled is None:
        v_tiled = torch.empty((g.B, g.H, shape.Lk, g.d), dtype=torch.bfloat16, device=k.device)
    if kbar is None and want_kbar:
        kbar = torch.empty((g.B, g.H, NK, g.d), dtype=torch.float32, device=k.device)
    _call("la_prep_kv_3d", ctypes.byref(g), _ptr(k), _ptr(v), ctypes.c_uint32(parts), _ptr(k_tiled), _ptr(v_tiled),
          _ptr(kbar), _stream(k))
    return k_tiled, v_tiled, kbar


def select_pooled(shape: Shape, qbar: torch.Tensor, kbar: torch.Tensor, tau: Optional[float] = None,
                  keep_blocks: Optional[int] = None, want_mask: bool = True, ws: Optional[torch.Tensor] = None):
    """Selection from pooled means (qbar fp32 [B,H,NQ,d], kbar fp32 [B,H,NK,d]) with the tau rule or
    the top-keep_blocks rule -> (mask, counts, idx) as select_blocks."""
    if (tau is None) == (keep_blocks is None):
        raise ValueError("give exactly one of tau and keep_blocks")
    B, H, d, block = shape.B, shape.H, shape.d, shape.block
    NQ, NK = nblocks(shape.Lq, block), nblocks(shape.Lk, block)
    for name, t, n in (("qbar", qbar, NQ), ("kbar", kbar, NK)):
        if t.device.type != "cuda" or t.dtype != torch.float32 or tuple(t.shape) != (B, H, n, d) \
                or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 {(B, H, n, d)} GPU tensor")
    mask = torch.empty((B, H, NQ, NK), dtype=torch.uint8, device=qbar.device) if want_mask else None
    counts = torch.empty((B, H, NQ), dtype=torch.int32, device=qbar.device)
    idx = torch.empty((B, H, NQ, NK), dtype=torch.int32, device=qbar.device)
    ws, nbytes = _workspace(shape, qbar.device, ws)
    if tau is not None:
        fn, arg = "la_select_pooled", ctypes.c_float(tau)
    else:
        fn, arg = "la_select_pooled_topk", ctypes.c_int32(keep_blocks)
    _call(fn, ctypes.byref(shape), _ptr(qbar), _ptr(kbar), arg, _ptr(mask), _ptr(counts), _ptr(idx), _ptr(ws),
          ctypes.c_size_t(nbytes), _stream(qbar))
    return mask, counts, idx


def untile_o_3d(g: Grid3D, o_tiled: torch.Tensor, lse_tiled: Optional[torch.Tensor] = None,
                o: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """Fused Untile Scatter: o_tiled [B,H,NQ block,d] (and lse_tiled) -> o linear [B,H,T_q Hs Ws,d] (and lse)."""
    shape = grid3d_shape(g)
    _check_lin("o_tiled", o_tiled, g, shape.Lq)
    L = g.T_q * g.Hs * g.Ws
    if o is None:
        o = torch.empty((g.B, g.H, L, g.d), dtype=torch.bfloat16, device=o_tiled.device)
    if lse is None and lse_tiled is not None:
        lse = torch.empty((g.B, g.H, L), dtype=torch.float32, device=o_tiled.device)
    _call("la_untile_o_3d", ctypes.byref(g), _ptr(o_tiled), _ptr(lse_tiled), _ptr(o), _ptr(lse), _stream(o_tiled))
    return o, lse


def bind_3d(g: Grid3D, q, k, v, q_t, k_t, v_t, qbar, kbar, mask, counts, idx, kvalid, o_t, lse_t, o, lse, ws,
            tau: Optional[float] = None, keep_blocks: Optional[int] = None, parts: int = LA_PART_ALL,
            scale: Optional[float] = None):
    """The 3-D path as BoundCalls on fixed tensors and the current stream:
    (prep_q, prep_kv, select, plan, run, merge, untile); in this order they compute what
    sparse_attn_3d computes."""
    if (tau is None) == (keep_blocks is None):
        raise ValueError("give exactly one of tau and keep_blocks")
    shape = grid3d_shape(g)
    st = _stream(q)
    nb = ctypes.c_size_t(ws.numel())
    keep = (g, shape, q, k, v, q_t, k_t, v_t, qbar, kbar, mask, counts, idx, kvalid, o_t, lse_t, o, lse, ws)
    gp, sp = ctypes.byref(g), ctypes.byref(shape)
    sc = ctypes.c_float(scale if scale is not None else 0.0)
    prep_q = BoundCall("la_prep_q_3d", gp, _ptr(q), _ptr(q_t), _ptr(qbar), st, keep=keep)
    prep_kv = BoundCall("la_prep_kv_3d", gp, _ptr(k), _ptr(v), ctypes.c_uint32(parts), _ptr(k_t), _ptr(v_t),
                        _ptr(kbar), st, keep=keep)
    if tau is not None:
        select = BoundCall("la_select_pooled", sp, _ptr(qbar), _ptr(kbar), ctypes.c_float(tau), _ptr(mask),
                           _ptr(counts), _ptr(idx), _ptr(ws), nb, st, keep=keep)
    else:
        select = BoundCall("la_select_pooled_topk", sp, _ptr(qbar), _ptr(kbar), ctypes.c_int32(keep_blocks),
                           _ptr(mask), _ptr(counts), _ptr(idx), _ptr(ws), nb, st, keep=keep)
    plan = BoundCall("la_sparse_attn_plan_valid", sp, _ptr(counts), _ptr(idx), _ptr(kvalid), _ptr(ws), nb, st,
                     keep=keep)
    run = BoundCall("la_sparse_attn_run", sp, _ptr(q_t), _ptr(k_t), _ptr(v_t), sc, _ptr(o_t), _ptr(lse_t), _ptr(ws),
                    nb, st, keep=keep)
    merge = BoundCall("la_sparse_attn_merge", sp, _ptr(o_t), _ptr(lse_t), _ptr(ws), nb, st, keep=keep)
    untile = BoundCall("la_untile_o_3d", gp, _ptr(o_t), _ptr(lse_t), _ptr(o), _ptr(lse), st, keep=keep)
    return prep_q, prep_kv, select, plan, run, merge, untile


def grid3d_positions(g: Grid3D, frames=None, device="cuda"):
    """Positions (frame, row, column) of the linear-order tokens of a grid, int32 [3, n]: (of the queries, of
    the keys).  frames: the positions of the T_ctx + T_q frames (retrieved frames need not be neighbours of the
    chunk); None numbers them from 0.  Text tokens have the position 0 on every axis (they are not turned)."""
    T = g.T_ctx + g.T_q
    f = torch.arange(T) if frames is None else torch.as_tensor(frames)
    if tuple(f.shape) != (T,):
        raise ValueError(f"frames must hold {T} positions")
    p = torch.stack(torch.meshgrid(f.to(torch.int32), torch.arange(g.Hs, dtype=torch.int32),
                                   torch.arange(g.Ws, dtype=torch.int32), indexing="ij")).flatten(1)
    k = torch.cat([torch.zeros((3, g.n_text), dtype=torch.int32), p], 1)
    return p[:, g.T_ctx * g.Hs * g.Ws:].contiguous().to(device), k.to(device)


class Rope(NamedTuple):
    """How a path turns its queries and keys (see rope): frequencies, pairs of each axis, and positions.
    Pairs are neighbours (2 j, 2 j + 1) unless interleaved is False, which is rope()'s own default."""
    freqs: torch.Tensor
    sections: Tuple[int, ...]
    q_positions: torch.Tensor
    k_positions: torch.Tensor
    interleaved: bool = True
    amplitude: float = 1.0


def sparse_attn_3d(g: Grid3D, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, tau: Optional[float] = None,
                   keep_blocks: Optional[int] = None, scale: Optional[float] = None, want_lse: bool = False,
                   kvalid: Optional[torch.Tensor] = None, rotary: Optional[Rope] = None):
    """The whole 3-D path on linear-order inputs: Q-Prep, KV-Prep, selection from the pooled means,
    attention over the tiled buffers with the padding masked, Untile Scatter.  rotary: q and k are turned by
    their positions first (grid3d_positions).  Returns (o linear, lse linear or None, mask over the tiled
    blocks, counts, idx)."""
    shape = grid3d_shape(g)
    if rotary is not None:
        q = rope(q, rotary.q_positions, rotary.freqs, interleaved=rotary.interleaved, sections=rotary.sections,
                 amplitude=rotary.amplitude)
        k = rope(k, rotary.k_positions, rotary.freqs, interleaved=rotary.interleaved, sections=rotary.sections,
                 amplitude=rotary.amplitude)
    if kvalid is None:
        kvalid = torch.from_numpy(grid3d_valid(g)[1]).to(q.device)
    q_t, qbar = prep_q_3d(g, q)
    k_t, v_t, kbar = prep_kv_3d(g, k, v)
    ws, _ = _workspace(shape, q.device, None)
    mask, counts, idx = select_pooled(shape, qbar, kbar, tau=tau, keep_blocks=keep_blocks, ws=ws)
    res = sparse_attn_fwd(q_t, k_t, v_t, counts, idx, g.block, scale=scale, n_text=shape.n_text, want_lse=want_lse,
                          ws=ws, kvalid=kvalid)
    o_t, lse_t = res if want_lse else (res, None)
    o, lse = untile_o_3d(g, o_t, lse_t)
    return o, lse, mask, counts, idx


# ----------------------------------------------------------------------------------------------
# rotary positions

LA_DTYPE_F32, LA_DTYPE_BF16 = 0, 1
_DTYPES = {torch.float32: LA_DTYPE_F32, torch.bfloat16: LA_DTYPE_BF16}


def rope_frequencies(rot: int, base: float = 10000.0, sections: Optional[Tuple[int, ...]] = None,
                     scaling: Optional[str] = None, factor: float = 1.0, trained: int = 0, turns=(1.0, 32.0),
                     device="cuda") -> torch.Tensor:
    """Radians per position of the rot / 2 pairs, float64: base^(-2 j / rot), or with `sections` (the pairs of
    each axis, adding up to rot / 2) a ladder base^(-i / n) of its own for every axis of n pairs.

    scaling  for contexts `factor` times as long as the trained ones:
      "linear"  every frequency divided by factor (positions interpolated);
      "base"    base multiplied by factor^(rot / (rot - 2)): the slowest pair is interpolated, the fastest kept;
      "ramp"    pairs that make fewer than turns[0] turns over the `trained` positions are interpolated, those of
                more than turns[1] are kept, and between them the two are mixed linearly in the turns."""
    if rot < 2 or rot % 2:
        raise ValueError("rot must be a positive even number")
    if base <= 0 or factor <= 0:
        raise ValueError("base and factor must be positive")
    if scaling == "base":
        if rot == 2 or sections is not None:
            raise ValueError("base scaling needs one axis of more than one pair")
        base = base * factor ** (rot / (rot - 2))
    parts = tuple(sections) if sections is not None else (rot // 2,)
    if sum(parts) != rot // 2 or min(parts) < 0:
        raise ValueError("sections must add up to rot / 2")
    f = torch.cat([float(base) ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in parts])
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        if trained < 1 or not turns[0] < turns[1]:
            raise ValueError("ramp scaling needs the trained length, and turns in ascending order")
        keep = ((trained * f / 6.283185307179586 - turns[0]) / (turns[1] - turns[0])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    elif scaling not in (None, "base"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return f.to(device)


def _rope_rows(name, t, like=None):
    """((B, L, H, d), (batch, token, head) strides) of [tokens, heads, d] or [B, heads, L, d] rows."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    n = t.dim()
    if t.dtype not in _DTYPES or (n != 3 and n != 4):
        raise TypeError(f"{name} must be a float32 or bfloat16 [tokens, heads, d] or [B, heads, L, d] tensor")
    if like is not None and (n != like.dim() or t.dtype is not like.dtype or t.get_device() != like.get_device()):
        raise ValueError(f"{name} differs in form, type or device from q")
    if n == 3:
        (L, H, d), B, (st, sh, sd), sb = t.shape, 1, t.stride(), 8
    else:
        (B, H, L, d), (sb, sh, st, sd) = t.shape, t.stride()
    # strides of an extent of one mean nothing
    if B <= 1:
        sb = 8
    if L <= 1:
        st = 8
    if H <= 1:
        sh = 8
    if (sd != 1 or (sb | st | sh) % 8) and B * L * H * d:
        raise ValueError(f"{name} must have contiguous rows, and strides that are multiples of 8")
    return (B, L, H, d), (sb, st, sh)


def rope(q: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, k: Optional[torch.Tensor] = None,
         interleaved: bool = False, sections: Optional[Tuple[int, ...]] = None, amplitude: float = 1.0,
         out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Queries (and keys) turned by their tokens' positions -> the same shape and type (a pair with k).

    q, k  bf16 or fp32, [tokens, heads, d] or [B, heads, L, d], any strides that are multiples of 8.
    positions  int32 [tokens] (or [L], shared by the batch), or with sections [axes, tokens]: the pairs of
    each axis, e.g. those of (frame, row, column).  freqs  float64 [rot / 2] (rope_frequencies): the first rot
    values of a head are turned, the others copied.  interleaved: pairs (2 j, 2 j + 1) instead of
    (j, j + rot / 2).  out and k_out may be q and k."""
    qshape, qs = _rope_rows("q", q)
    B, L, Hq, d = qshape
    packed = q.dim() == 3
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        os = (8, max(Hq, 1) * d, d) if packed else (Hq * L * d, d, max(L, 1) * d)
    else:
        oshape, os = _rope_rows("out", out, q)
        if oshape != qshape:
            raise ValueError(f"out has shape {tuple(out.shape)}, q has {tuple(q.shape)}")
    Hk, ks, kos = 0, (0, 0, 0), (0, 0, 0)
    if k is not None:
        kshape, ks = _rope_rows("k", k, q)
        Hk = kshape[2]
        if kshape != (B, L, Hk, d):
            raise ValueError(f"k has shape {tuple(k.shape)}, q has {tuple(q.shape)}")
        if k_out is None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
            kos = (8, max(Hk, 1) * d, d) if packed else (Hk * L * d, d, max(L, 1) * d)
        else:
            koshape, kos = _rope_rows("k_out", k_out, q)
            if koshape != kshape:
                raise ValueError(f"k_out has shape {tuple(k_out.shape)}, k has {tuple(k.shape)}")
    axes = 1 if sections is None else len(sections)
    dev = q.get_device()
    if not isinstance(freqs, torch.Tensor) or freqs.get_device() != dev or freqs.dtype is not torch.float64 \
            or freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError(f"freqs must be a contiguous float64 [rot / 2] tensor on {q.device}")
    pairs = freqs.shape[0]
    if not 1 <= axes <= 3 or (sections is not None and sum(sections) != pairs):
        raise ValueError("sections must be the pairs of one to three axes, rot / 2 in all")
    _check_ints("positions", positions, dev, (L,) if sections is None else (axes, L))
    shape = RopeShape(B, L, Hq, Hk, d, 2 * pairs, 1 if interleaved else 0, _DTYPES[q.dtype], axes,
                      (pairs,) if sections is None else tuple(sections), *qs, *os, *ks, *kos)
    _on_device(dev, "la_rope", ctypes.byref(shape), q.data_ptr(), out.data_ptr(), _ptr(k), _ptr(k_out),
               positions.data_ptr(), freqs.data_ptr(), amplitude, _stream(q))
    return out if k is None else (out, k_out)


# ----------------------------------------------------------------------------------------------
# packed sequences

def _rows(name, t: torch.Tensor, dev=None, heads=None, d=None, tokens=None):
    """(tokens, heads, d, token stride, head stride) of a bf16 GPU tensor [tokens, heads, d] with contiguous
    rows and strides that are multiples of 8; raises for anything else, and for another device, number of
    heads, head dimension or number of tokens than given.  The strides of an extent of one, which mean
    nothing, are given as a packed tensor's."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not torch.bfloat16 or t.dim() != 3:
        raise TypeError(f"{name} must be a bfloat16 [tokens, heads, d] tensor")
    if dev is not None and t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, other operands are on device {dev}")
    T, H, D = t.shape
    if (tokens is not None and T != tokens) or (heads is not None and H != heads) or (d is not None and D != d):
        raise ValueError(f"{name} has shape {(T, H, D)}, inconsistent with the other operands")
    st, sh, sd = t.stride()
    if H <= 1:
        sh = D
    if T <= 1:
        st = max(H, 1) * D
    if (sd != 1 or (st | sh) % 8) and T * H * D:
        raise ValueError(f"{name} must have contiguous rows, and strides that are multiples of 8")
    return T, H, D, st, sh


def _check_ints(name, t: torch.Tensor, dev, shape):
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.int32 or t.shape != shape or t.get_device() != dev \
            or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 {list(shape)} tensor on GPU {dev}")


# 0.1 us; torch.cuda.current_device() looks whether CUDA is initialised first and takes 0.5
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_device(dev: int, fn: str, *args):
    """_call with device `dev` as the current one (the launches go there)."""
    if _current_device() == dev:
        _call(fn, *args)
    else:
        with torch.cuda.device(dev):
            _call(fn, *args)


def _seqs(S, Tq, Tk, Hq, Hkv, *rest):
    """A la_seqs by reference; ctypes would drop what passes 32 bits."""
    if max(S, Tq, Tk, Hq, Hkv) > 0x7fffffff:
        raise ValueError("2^31 or more sequences, tokens or heads")
    return ctypes.byref(Seqs(S, Tq, Tk, Hq, Hkv, *rest))


def _outputs(q, dev, T, Hq, d, want_lse, out, lse_out):
    """(o, its token and head stride, lse or None)."""
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        st, sh = Hq * d, d
    else:
        _, _, _, st, sh = _rows("out", out, dev, Hq, d, T)
    if lse_out is None:
        if want_lse:
            lse_out = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
    elif lse_out.dtype is not torch.float32 or lse_out.shape != (T, Hq) or not lse_out.is_contiguous() \
            or lse_out.get_device() != dev:
        raise ValueError(f"lse_out must be a contiguous float32 {[T, Hq]} tensor on GPU {dev}")
    return out, st, sh, lse_out


def _scratch(need, q, dev, ws):
    """(pointer, bytes, tensor) of the workspace of a call that needs `need` bytes."""
    if ws is None:
        if need == 0:
            return None, 0, None
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
        return ws.data_ptr(), need, ws
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous tensor on GPU {dev}")
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def prompt_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor,
                cu_k: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None,
                want_lse: bool = False, ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                lse_out: Optional[torch.Tensor] = None):
    """Attention of packed sequences over their own keys -> o bf16 [Tq, Hq, d] (and lse fp32 [Tq, Hq]).

    q [Tq, Hq, d]; k, v [Tk, Hkv, d] in bf16, Hq a multiple of Hkv; token and head strides are free
    (multiples of 8).  cu_q, cu_k int32 [S + 1] on the GPU: the first row of every sequence (cu_k None:
    cu_q).  Causal: the last query of a sequence sees its last key.  Rows behind the last sequence are
    not written (a new output holds anything there)."""
    Tq, Hq, d, qt, qh = _rows("q", q)
    dev = q.get_device()
    Tk, Hkv, _, kt, kh = _rows("k", k, dev, d=d)
    _, _, _, vt, vh = _rows("v", v, dev, Hkv, d, Tk)
    if cu_k is None:
        cu_k = cu_q
    S = cu_q.numel() - 1 if isinstance(cu_q, torch.Tensor) else 0
    _check_ints("cu_q", cu_q, dev, (S + 1,))
    _check_ints("cu_k", cu_k, dev, (S + 1,))
    o, ot, oh, lse = _outputs(q, dev, Tq, Hq, d, want_lse, out, lse_out)
    seqs = _seqs(S, Tq, Tk, Hq, Hkv, d, 1 if causal else 0, qt, qh, ot, oh, kt, kh, vt, vh)
    wp, nbytes, ws = _scratch(lib().la_prompt_ws_bytes(seqs), q, dev, ws)
    _on_device(dev, "la_prompt_attn", seqs, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(),
               scale if scale is not None else 0.0, o.data_ptr(), _ptr(lse), wp, nbytes, _stream(q))
    return o if lse is None else (o, lse)


def kv4_cache(n_pages: int, Hkv: int, d: int, page: int = 64, device="cuda") -> torch.Tensor:
    """An empty 4-bit cache: uint8 [n_pages, Hkv, page (d + d / 16)], `page` tokens to a page (a power of
    two, 16 to 1024)."""
    nbytes = int(lib().la_kv4_page_bytes(d, page))
    if nbytes == 0:
        raise ValueError(f"no 4-bit cache for d = {d} and pages of {page} tokens")
    return torch.zeros((n_pages, Hkv, nbytes), dtype=torch.uint8, device=device)


def _check_cache(cache, lens, table, cu, d):
    """(key heads, the la_kv4 of a cache and its table, sequences); raises for what does not fit."""
    if not isinstance(cache, torch.Tensor) or not cache.is_cuda:
        raise TypeError("cache must be a GPU tensor")
    if cache.dtype is not torch.uint8 or cache.dim() != 3 or not cache.is_contiguous():
        raise TypeError("cache must be a contiguous uint8 [n_pages, Hkv, page bytes] tensor")
    n, Hkv, nbytes = cache.shape
    page, rest = divmod(nbytes, d + d // 16) if d > 0 else (0, 0)
    if rest or page < 16 or page & (page - 1):
        raise ValueError(f"a cache of {nbytes} bytes a page is none for heads of {d}")
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table must be an int32 [S, max_pages] tensor")
    dev = cache.get_device()
    S, most = table.shape
    if most > 0x7fffffff:
        raise ValueError("2^31 or more pages to a sequence")
    _check_ints("table", table, dev, (S, most))
    _check_ints("lens", lens, dev, (S,))
    _check_ints("cu", cu, dev, (S + 1,))
    return Hkv, ctypes.byref(Kv4(n, page, most)), S


def kv4_append(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, lens: torch.Tensor,
               table: torch.Tensor) -> None:
    """Enters k, v (bf16 [T, Hkv, d], free strides) into a 4-bit cache: rows [cu[s], cu[s + 1]) are the
    last tokens of sequence s, which has lens[s] with them, on the pages table[s].  cu int32 [S + 1],
    lens int32 [S], table int32 [S, max_pages], all on the GPU."""
    T, H, d, kt, kh = _rows("k", k)
    dev = k.get_device()
    _, _, _, vt, vh = _rows("v", v, dev, H, d, T)
    Hkv, kv, S = _check_cache(cache, lens, table, cu, d)
    if cache.get_device() != dev or Hkv != H:
        raise ValueError(f"cache of {Hkv} heads on {cache.device}, k of {H} on {k.device}")
    _on_device(dev, "la_kv4_append", _seqs(S, 0, T, H, H, d, 0, 0, 0, 0, 0, kt, kh, vt, vh), kv, k.data_ptr(),
               v.data_ptr(), cu.data_ptr(), lens.data_ptr(), table.data_ptr(), cache.data_ptr(), _stream(k))


def kv4_read(cache: torch.Tensor, cu: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, tokens: int, d: int,
             out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
    """The values that the last cu[s + 1] - cu[s] tokens of every sequence stand for -> (k, v) bf16
    [tokens, Hkv, d] (or the given pair, of any strides): what kv4_append entered there, rounded."""
    H, kv, S = _check_cache(cache, lens, table, cu, d)
    dev = cache.get_device()
    if out is None:
        k, v = torch.empty((2, tokens, H, d), dtype=torch.bfloat16, device=cache.device).unbind(0)
        kt = vt = H * d
        kh = vh = d
    else:
        k, v = out
        _, _, _, kt, kh = _rows("k", k, dev, H, d, tokens)
        _, _, _, vt, vh = _rows("v", v, dev, H, d, tokens)
    _on_device(dev, "la_kv4_read", _seqs(S, 0, tokens, H, H, d, 0, 0, 0, 0, 0, kt, kh, vt, vh), kv,
               cache.data_ptr(), cu.data_ptr(), lens.data_ptr(), table.data_ptr(), k.data_ptr(), v.data_ptr(),
               _stream(cache))
    return k, v


def kv4_attn(q: torch.Tensor, cache: torch.Tensor, cu_q: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
             max_q: int, causal: bool = True, scale: Optional[float] = None, want_lse: bool = False,
             ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             lse_out: Optional[torch.Tensor] = None):
    """Attention of packed queries over a 4-bit cache -> o bf16 [Tq, Hq, d] (and lse fp32 [Tq, Hq]).

    q [Tq, Hq, d] in bf16 with free strides; sequence s has the rows [cu_q[s], cu_q[s + 1]), at most max_q
    of them (1: the next token of every sequence), and lens[s] tokens in the cache (see kv4_append).  Rows of
    a sequence that has more than max_q, and rows behind the last sequence, are not written (a new output
    holds anything there).  Causal: the last query of a sequence sees the last token, its queries being the
    last tokens."""
    Tq, Hq, d, qt, qh = _rows("q", q)
    dev = q.get_device()
    Hkv, kv, S = _check_cache(cache, lens, table, cu_q, d)
    if cache.get_device() != dev:
        raise ValueError(f"cache is on {cache.device}, q on {q.device}")
    o, ot, oh, lse = _outputs(q, dev, Tq, Hq, d, want_lse, out, lse_out)
    seqs = _seqs(S, Tq, 0, Hq, Hkv, d, 1 if causal else 0, qt, qh, ot, oh, 0, 0, 0, 0)
    max_q = min(max(max_q, -1), Tq)            # a c_int32; below 0 it is refused
    wp, nbytes, ws = _scratch(lib().la_kv4_ws_bytes(seqs, kv, max_q), q, dev, ws)
    _on_device(dev, "la_kv4_attn", seqs, kv, max_q, q.data_ptr(), cache.data_ptr(), cu_q.data_ptr(), lens.data_ptr(),
               table.data_ptr(), scale if scale is not None else 0.0, o.data_ptr(), _ptr(lse), wp, nbytes, _stream(q))
    return o if lse is None else (o, lse)


# ----------------------------------------------------------------------------------------------
# scalar policy (Sec. 3.1, Sec. 3.2)

LATENT_MSE_WS_BYTES = 8192


def latent_mse(z_a: torch.Tensor, z_b: torch.Tensor, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """D_t = MSE(z_a, z_b) over every value (fp32 or bf16 GPU tensors of one shape) -> float64
    GPU tensor of one element."""
    for name, t in (("z_a", z_a), ("z_b", z_b)):
        if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous GPU tensor")
    if z_a.dtype != z_b.dtype or z_a.shape != z_b.shape:
        raise ValueError("z_a and z_b must have one dtype and one shape")
    dt = {torch.float32: LA_DTYPE_F32, torch.bfloat16: LA_DTYPE_BF16}.get(z_a.dtype)
    if dt is None:
        raise TypeError("latents must be float32 or bfloat16")
    if ws is None:
        ws = torch.empty(LATENT_MSE_WS_BYTES, dtype=torch.uint8, device=z_a.device)
    if out is None:
        out = torch.empty(1, dtype=torch.float64, device=z_a.device)
    _call("la_latent_mse", _ptr(z_a), _ptr(z_b), ctypes.c_int64(z_a.numel()), ctypes.c_int32(dt), _ptr(out),
          _ptr(ws), ctypes.c_size_t(ws.numel()), _stream(z_a))
    return out


def dynamics_ema(D_t: float, D_bar_prev: Optional[float], alpha: float) -> float:
    """D_bar_t = alpha D_t + (1 - alpha) D_bar_{t-1}; None starts the average (host only)."""
    res = ctypes.c_double()
    prev = None if D_bar_prev is None else ctypes.byref(ctypes.c_double(D_bar_prev))
    _call("la_dynamics_ema", ctypes.c_double(D_t), prev, ctypes.c_double(alpha), ctypes.byref(res))
    return res.value


def temporal_window(D_bar: float, kappa: float, L_m: int) -> int:
    """L_t = clip(floor(L_m kappa / (D_bar + kappa)), 1, L_m) (host only)."""
    res = ctypes.c_int32()
    _call("la_temporal_window", ctypes.c_double(D_bar), ctypes.c_double(kappa), ctypes.c_int32(L_m),
          ctypes.byref(res))
    return res.value


def pose_revisiting(similarities, tau_pose: float) -> bool:
    """max_j similarities[j] >= tau_pose (host only; float32 comparisons)."""
    import numpy as np
    sims = np.ascontiguousarray(similarities, dtype=np.float32)
    res = ctypes.c_int32()
    _call("la_pose_revisiting", sims.ctypes.data_as(_P) if sims.size else None, ctypes.c_int32(sims.size),
          ctypes.c_float(tau_pose), ctypes.byref(res))
    return bool(res.value)


def denoise_schedule(K: int, reuse: bool):
    """For each of the K denoising steps, the step whose model output it uses (host only)."""
    import numpy as np
    src = np.zeros(max(K, 1), dtype=np.int32)
    _call("la_denoise_schedule", ctypes.c_int32(K), ctypes.c_int32(1 if reuse else 0), src.ctypes.data_as(_P))
    return [int(x) for x in src[:K]]


def bf16_from_bits(bits, device="cuda") -> torch.Tensor:
    """uint16 numpy array of bfloat16 bit patterns -> bfloat16 tensor on `device` (no rounding)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    return t.to(device)
