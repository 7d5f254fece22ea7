"""Python binding of the layer operators of libpspo (include/pspo_layer.h): argument marshalling only.

The token-wise operators of a policy's transformer layers on packed prefix tokens: the norms of
queries and keys with the position rotation, dropout with the residual sum, and the gated
feed-forward block, each with its gradient.  As in ``pspo``: every step runs in the HIP kernels of
libpspo.so on the current stream, tensors must be on the current device, a missing library raises.
All calls take the first N rows of their per-token tensors and leave the rows behind them (of given
outputs) as they were.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import pspo
from .pspo import _dev

TYPE_BF16, TYPE_F32 = 0, 1
ROPE_INTERLEAVED, QK_NO_NORM = 1, 2
ACTIVATIONS = {"silu": 0, "gelu_tanh": 1}
FFN_DW_F32, FFN_BACKWARD, FFN_PREACT = 256, 512, 1024

_P = ctypes.c_void_p
_I32, _I64, _U32, _U64, _F32, _F64, _SZ = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64,
                                           ctypes.c_float, ctypes.c_double, ctypes.c_size_t)

_SIGNATURES = {
    "pspo_qk_norm_rope_fwd": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _I32, _I32, _I32, _I32,
                                             _I32, _I32, _F32, _I32, _U32, _P, _P, _P, _P]),
    "pspo_qk_norm_rope_workspace_bytes": (_SZ, [_I32, _I32]),
    "pspo_qk_norm_rope_bwd": (ctypes.c_int, [_P, _P, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _I32, _I32, _I32,
                                             _I32, _I32, _I32, _F32, _I32, _U32, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "pspo_dropout_add_fwd": (ctypes.c_int, [_P, _P, _P, _I32, _I32, _F64, _U64, _U64, _I32, _P, _P]),
    "pspo_gated_ffn_workspace_bytes": (_SZ, [_I32, _I32, _I32, _U32]),
    "pspo_gated_ffn_fwd": (ctypes.c_int, [_P, _P, _P, _P, _I32, _I32, _I32, _I32, _P, _P, _P, _SZ, _P]),
    "pspo_gated_ffn_bwd": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _U32, _P, _P, _P, _P, _P,
                                          _SZ, _P]),
    "pspo_dropout_bwd": (ctypes.c_int, [_P, _P, _I32, _I32, _F64, _U64, _U64, _I32, _I32, _P, _P]),
}

_lib = None


# The calls are short next to a Python call's own cost (5 us and up), so a tensor is looked at
# with the cheap queries first, and pspo._dev runs for what they find wrong, to say what.

def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _here(t, dtype, name: str, device: int) -> None:
    """t: a contiguous tensor of `dtype` on the current device (`device`)."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _dev(t, dtype, name)


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _check(rc: int) -> None:
    if rc:
        pspo._check(rc)


def load() -> ctypes.CDLL:
    """libpspo.so with the signatures of the layer operators; raises if it is missing."""
    global _lib
    if _lib is None:
        lib = pspo.load()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def exported_symbols():
    return list(_SIGNATURES)


def _type(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype == torch.bfloat16:
        return TYPE_BF16
    if t.dtype == torch.float32:
        return TYPE_F32
    raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")


def _rows(t: torch.Tensor, N: int, shape, name: str) -> None:
    """t must be [>= N, *shape]."""
    have = t.shape if isinstance(t, torch.Tensor) else ()
    if len(have) != 1 + len(shape) or have[1:] != shape or have[0] < N:
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        raise ValueError(f"{name} must be [>= {N}{''.join(', %d' % s for s in shape)}], got {list(t.shape)}")


def _exact(t: torch.Tensor, shape, name: str) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _apart(out: torch.Tensor, name: str, *others, used: Optional[int] = None) -> None:
    """`out` (its first `used` bytes, if given) must not share memory with the call's other tensors."""
    size = out.numel() * out.element_size()
    if used is not None and used < size:
        size = used
    if size == 0:
        return
    lo = out.data_ptr()
    hi = lo + size
    for t in others:
        if t is None or t.numel() == 0:
            continue
        at = t.data_ptr()
        if at >= hi:
            continue
        last = t.numel() - 1 if t.is_contiguous() else sum((s - 1) * st for s, st in zip(t.shape, t.stride()))
        if at + (last + 1) * t.element_size() > lo:
            raise ValueError(f"{name} overlaps an input or another output")


def _ints(t: Optional[torch.Tensor], n: int, name: str, device: int) -> None:
    if t is None:
        return
    _here(t, torch.int32, name, device)
    if t.dim() != 1 or t.shape[0] < n:
        raise ValueError(f"{name} must be [>= {n}], got {list(t.shape)}")


_MOST = 2 ** 31 - 1   # the C calls take 32-bit counts, and ctypes passes the low bits of a larger number


def _fits(n: int, name: str) -> int:
    if n > _MOST:
        raise ValueError(f"{name} must be at most {_MOST}, got {n}")
    return n


def _count(N: int) -> int:
    if N < 0:
        raise ValueError("N must be >= 0")
    N = int(N)
    return N if N <= _MOST else _fits(N, "N")


# ---------------------------------------------------------------------------
# norms of queries and keys with the position rotation
# ---------------------------------------------------------------------------

def _heads(t: torch.Tensor, N: int, name: str, device: int, like: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[>= N, heads, D] on the current device, heads contiguous, any row stride."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be a tensor [>= N, heads, head_dim]")
    if t.shape[0] < N:
        raise ValueError(f"{name} has fewer than N rows")
    if t.get_device() != device:
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        raise ValueError(f"{name} is on {t.device}, but the calls run on the current device cuda:{device}")
    if like is not None and t.dtype != like.dtype:
        raise TypeError(f"{name} must have dtype {like.dtype}, got {t.dtype}")
    _, H, D = t.shape
    if H > _MOST or D > _MOST:
        _fits(max(H, D), f"heads and head_dim of {name}")
    if (D > 1 and t.stride(2) != 1) or (H > 1 and t.stride(1) != D):
        raise ValueError(f"the heads of {name} must be contiguous within a row")
    return t


def _row_stride(t: Optional[torch.Tensor]) -> int:
    """Elements between rows (a tensor of one row may report any stride)."""
    if t is None:
        return 0
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _qk_common(q, k, q_weight, k_weight, inv_freq, N, positions, seq_id, cu_seqlens, first_pos, interleaved, norm,
               err_flag):
    device = torch.cuda.current_device()
    ty = _type(q, "q")
    _heads(q, N, "q", device)
    D = q.shape[2]
    if k is not None:
        _heads(k, N, "k", device, q)
        if k.shape[2] != D:
            raise ValueError("q and k disagree on the head dimension")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _here(w, q.dtype, name, device)
            _exact(w, (D,), name)
    rot, R = 0, 0
    if inv_freq is not None:
        _here(inv_freq, torch.float32, "inv_freq", device)
        if inv_freq.dim() != 1:
            raise ValueError("inv_freq must be [rot_dim / 2]")
        rot = 2 * inv_freq.shape[0]
        if rot > _MOST:
            _fits(rot, "rot_dim")
        if positions is not None:
            _ints(positions, N, "positions", device)
            seq_id = cu_seqlens = first_pos = None
        else:
            if seq_id is None or cu_seqlens is None:
                raise ValueError("positions, or seq_id and cu_seqlens, must be given")
            _ints(seq_id, N, "seq_id", device)
            _ints(cu_seqlens, 1, "cu_seqlens", device)
            R = _fits(cu_seqlens.shape[0] - 1, "R")
            _ints(first_pos, R, "first_pos", device)
    else:
        positions = seq_id = cu_seqlens = first_pos = None
    if err_flag is not None:
        _here(err_flag, torch.int32, "err_flag", device)
    flags = (ROPE_INTERLEAVED if interleaved else 0) | (0 if norm else QK_NO_NORM)
    heads = (N, R, q.shape[1], 0 if k is None else k.shape[1], D, rot)
    ins = (q.data_ptr(), _ptr(k), _row_stride(q), _row_stride(k), _ptr(q_weight), _ptr(k_weight), _ptr(inv_freq),
           _ptr(positions), _ptr(seq_id), _ptr(cu_seqlens), _ptr(first_pos))
    read = (q, k, q_weight, k_weight, inv_freq, positions, seq_id, cu_seqlens, first_pos, err_flag)
    return device, ty, D, flags, ins, heads, read


def qk_norm_rope(q, k, q_weight, k_weight, inv_freq, N: int, positions=None, seq_id=None, cu_seqlens=None,
                 first_pos=None, eps: float = 1e-6, interleaved: bool = False, norm: bool = True,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                 err_flag: Optional[torch.Tensor] = None) -> dict:
    """Head norms and position rotation of the first N rows of q [>=N, Hq, D] and k [>=N, Hk, D] (or None).

    bf16 or float32; the rows may be strided (parts of a fused projection), the heads of a row
    contiguous.  q_weight, k_weight: [D] of the same type or None (ones).  inv_freq: float32
    [rot / 2] (None: no rotation), the first `rot` entries of a head are turned.  Positions: int32
    [N], or from the packer's seq_id and cu_seqlens plus each completion's first position.
    Returns q and k ([N, H, D] contiguous; k None if there is none).
    """
    N = _count(N)
    device, ty, D, flags, ins, heads, read = _qk_common(q, k, q_weight, k_weight, inv_freq, N, positions, seq_id,
                                                        cu_seqlens, first_pos, interleaved, norm, err_flag)
    outs = []
    for name, x, o in (("q_out", q, q_out), ("k_out", k, k_out)):
        if x is None:
            if o is not None:
                raise ValueError(f"{name} is given without its input")
            outs.append(None)
            continue
        if o is None:
            o = torch.empty((N, x.shape[1], D), dtype=x.dtype, device=x.device)
        else:
            _rows(o, N, (x.shape[1], D), name)
            _here(o, x.dtype, name, device)
            _apart(o, name, *read, *outs)
        outs.append(o)
    qo, ko = outs
    _check((_lib or load()).pspo_qk_norm_rope_fwd(*ins, *heads, eps, ty, flags, qo.data_ptr(), _ptr(ko),
                                                  _ptr(err_flag), _stream(device)))
    if q_out is not None:
        qo = qo[:N]
    if k_out is not None:
        ko = ko[:N]
    return dict(q=qo, k=ko)


def qk_norm_rope_bwd(dq_out, dk_out, q, k, q_weight, k_weight, inv_freq, N: int, positions=None, seq_id=None,
                     cu_seqlens=None, first_pos=None, eps: float = 1e-6, interleaved: bool = False, norm: bool = True,
                     want_weights: bool = True, workspace: Optional[torch.Tensor] = None,
                     err_flag: Optional[torch.Tensor] = None) -> dict:
    """Gradient of qk_norm_rope from its inputs and the gradients of its outputs ([>=N, H, D] contiguous).

    Returns dq, dk ([N, H, D] contiguous, of the inputs' type) and, for the weights that are given
    (unless want_weights is False), dq_weight and dk_weight (float32 [D]).
    """
    N = _count(N)
    device, ty, D, flags, ins, heads, read = _qk_common(q, k, q_weight, k_weight, inv_freq, N, positions, seq_id,
                                                        cu_seqlens, first_pos, interleaved, norm, err_flag)
    if (k is None) != (dk_out is None):
        raise ValueError("k and dk_out must be both given or both None")
    dx = []
    for name, x, g in (("dq_out", q, dq_out), ("dk_out", k, dk_out)):
        if x is None:
            dx.append(None)
            continue
        _rows(g, N, (x.shape[1], D), name)
        _here(g, x.dtype, name, device)
        dx.append(torch.empty((N, x.shape[1], D), dtype=x.dtype, device=x.device))
    dw = [torch.empty(D, dtype=torch.float32, device=q.device) if w is not None and want_weights else None
          for w in (q_weight, k_weight)]
    lib = _lib or load()
    if workspace is not None:
        _here(workspace, torch.uint8, "workspace", device)
    if dw[0] is not None or dw[1] is not None:
        need = lib.pspo_qk_norm_rope_workspace_bytes(N, D)
        if workspace is None:
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
        else:
            _apart(workspace, "workspace", *read, dq_out, dk_out, used=need)
    _check(lib.pspo_qk_norm_rope_bwd(
        dq_out.data_ptr(), _ptr(dk_out), *ins, *heads, eps, ty, flags, dx[0].data_ptr(), _ptr(dx[1]), _ptr(dw[0]),
        _ptr(dw[1]), _ptr(err_flag), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(device)))
    return dict(dq=dx[0], dk=dx[1], dq_weight=dw[0], dk_weight=dw[1], workspace=workspace)


# ---------------------------------------------------------------------------
# dropout with the residual sum
# ---------------------------------------------------------------------------

_U64_MASK = 2 ** 64 - 1


def dropout_add(x, N: int, p: float, seed: int, offset: int = 0, residual: Optional[torch.Tensor] = None,
                row_ids: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x) of the first N rows of x [>=N, d] (bf16 or float32); no mask is stored.

    An entry is kept with probability T / 2^16, T = floor((1 - p) 2^16 + 1/2), and scaled by its inverse.
    The mask depends on (seed, offset, column, row_ids[n]) only (row_ids None: the row itself); with
    the packer's src_row it is the same for every draw of the cutoffs.  Returns [N, d].
    """
    N = _count(N)
    device = torch.cuda.current_device()
    ty = _type(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [>= N, d]")
    d = _fits(x.shape[1], "d")
    _rows(x, N, (d,), "x")
    _here(x, x.dtype, "x", device)
    if residual is not None:
        _rows(residual, N, (d,), "residual")
        _here(residual, x.dtype, "residual", device)
    _ints(row_ids, N, "row_ids", device)
    if out is None:
        out = torch.empty((N, d), dtype=x.dtype, device=x.device)
    else:
        _rows(out, N, (d,), "out")
        _here(out, x.dtype, "out", device)
        _apart(out, "out", x, residual, row_ids)
    _check((_lib or load()).pspo_dropout_add_fwd(x.data_ptr(), _ptr(residual), _ptr(row_ids), N, d, p, seed & _U64_MASK,
                                                 offset & _U64_MASK, ty, out.data_ptr(), _stream(device)))
    return out if out.shape[0] == N else out[:N]


def dropout_bwd(dy, N: int, p: float, seed: int, offset: int = 0, row_ids: Optional[torch.Tensor] = None,
                out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of dropout_add to x (the residual's is dy itself): the mask drawn again and applied to dy.

    dy: [>=N, d] bf16 or float32 (e.g. the loss call's d_hidden); the result is of out_dtype (default: dy's).
    """
    N = _count(N)
    device = torch.cuda.current_device()
    ty = _type(dy, "dy")
    if dy.dim() != 2:
        raise ValueError("dy must be [>= N, d]")
    d = _fits(dy.shape[1], "d")
    _rows(dy, N, (d,), "dy")
    _here(dy, dy.dtype, "dy", device)
    _ints(row_ids, N, "row_ids", device)
    if out is None:
        out = torch.empty((N, d), dtype=out_dtype or dy.dtype, device=dy.device)
    else:
        _rows(out, N, (d,), "out")
        _here(out, out_dtype or out.dtype, "out", device)
        _apart(out, "out", dy, row_ids)
    _check((_lib or load()).pspo_dropout_bwd(dy.data_ptr(), _ptr(row_ids), N, d, p, seed & _U64_MASK,
                                             offset & _U64_MASK, ty, _type(out, "out"), out.data_ptr(),
                                             _stream(device)))
    return out if out.shape[0] == N else out[:N]


# ---------------------------------------------------------------------------
# the gated feed-forward block
# ---------------------------------------------------------------------------

def _act(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return ACTIVATIONS[act]


def _ffn_weights(w_gate, w_up, w_down):
    device = torch.cuda.current_device()
    if not isinstance(w_gate, torch.Tensor):
        raise TypeError("w_gate must be a torch.Tensor")
    if w_gate.dim() != 2:
        raise ValueError("w_gate must be [f, d]")
    f, d = w_gate.shape
    if d > _MOST or f > _MOST:
        _fits(max(d, f), "d and f")
    _exact(w_up, (f, d), "w_up")
    _exact(w_down, (d, f), "w_down")
    for name, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _here(w, torch.bfloat16, name, device)
    return device, d, f


def gated_ffn_workspace_bytes(N: int, d: int, f: int, backward: bool = False, preact: bool = False) -> int:
    """Bytes of workspace that gated_ffn (gated_ffn_bwd; with kept pre-activations) takes for up to N tokens."""
    flags = (FFN_BACKWARD if backward else 0) | (FFN_PREACT if preact else 0)
    return int(load().pspo_gated_ffn_workspace_bytes(_fits(N, "N"), _fits(d, "d"), _fits(f, "f"), flags))


def _ffn_workspace(workspace, N, d, f, flags, like, device, *others):
    need = (_lib or load()).pspo_gated_ffn_workspace_bytes(N, d, f, flags)
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
    _here(workspace, torch.uint8, "workspace", device)
    _apart(workspace, "workspace", *others, used=need)
    return workspace


def gated_ffn(x, w_gate, w_up, w_down, N: int, act: str = "silu", keep: bool = False,
              out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T of the first N rows of x [>=N, d], all bf16.

    w_gate, w_up: [f, d]; w_down: [d, f]; act: "silu" or "gelu_tanh".  Returns y ([N, d]) and, with
    keep, the float32 pre-activations [N, 2 f] that gated_ffn_bwd takes (else preact is None).  The
    same call gives the same bits; a token's y may differ in rounding between calls of different N.
    """
    N = _count(N)
    kind = _act(act)
    device, d, f = _ffn_weights(w_gate, w_up, w_down)
    _rows(x, N, (d,), "x")
    _here(x, torch.bfloat16, "x", device)
    if out is None:
        out = torch.empty((N, d), dtype=torch.bfloat16, device=x.device)
    else:
        _rows(out, N, (d,), "out")
        _here(out, torch.bfloat16, "out", device)
        _apart(out, "out", x, w_gate, w_up, w_down)
    pre = torch.empty((N, 2 * f), dtype=torch.float32, device=x.device) if keep else None
    workspace = _ffn_workspace(workspace, N, d, f, 0, x, device, x, w_gate, w_up, w_down, out)
    _check((_lib or load()).pspo_gated_ffn_fwd(
        x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), N, d, f, kind, out.data_ptr(), _ptr(pre),
        workspace.data_ptr(), workspace.numel(), _stream(device)))
    return dict(y=out if out.shape[0] == N else out[:N], preact=pre, workspace=workspace)


def gated_ffn_bwd(dy, x, w_gate, w_up, w_down, N: int, act: str = "silu", preact: Optional[torch.Tensor] = None,
                  dw: Optional[tuple] = None, accumulate: bool = False,
                  workspace: Optional[torch.Tensor] = None) -> dict:
    """Gradient of gated_ffn: dx [N, d] (bf16), dw_gate, dw_up [f, d], dw_down [d, f].

    dy: bf16 [>=N, d]; preact: what gated_ffn kept (None: computed again).  dw: the three weight
    gradients to write, all bf16 or all float32 (None: bf16); accumulate adds to them (float32).
    """
    N = _count(N)
    kind = _act(act)
    device, d, f = _ffn_weights(w_gate, w_up, w_down)
    for name, t in (("dy", dy), ("x", x)):
        _rows(t, N, (d,), name)
        _here(t, torch.bfloat16, name, device)
    if preact is not None:
        _rows(preact, N, (2 * f,), "preact")
        _here(preact, torch.float32, "preact", device)
    shapes = ((f, d), (f, d), (d, f))
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs dw")
        dw = tuple(torch.empty(s, dtype=torch.bfloat16, device=x.device) for s in shapes)
    else:
        if len(dw) != 3:
            raise ValueError("dw must hold the three weight gradients")
        for i, (t, s, name) in enumerate(zip(dw, shapes, ("dw_gate", "dw_up", "dw_down"))):
            ty = _type(t, name)
            if ty != _type(dw[0], name):
                raise TypeError("the weight gradients must have one dtype")
            _exact(t, s, name)
            _here(t, t.dtype, name, device)
            _apart(t, name, dy, x, w_gate, w_up, w_down, preact, *dw[:i])
    flags = (FFN_DW_F32 if dw[0].dtype == torch.float32 else 0) | (pspo.PSPO_ACCUMULATE_DW if accumulate else 0)
    dx = torch.empty((N, d), dtype=torch.bfloat16, device=x.device)
    need = FFN_BACKWARD | (FFN_PREACT if preact is not None else 0)
    workspace = _ffn_workspace(workspace, N, d, f, need, x, device, dy, x, w_gate, w_up, w_down, preact, *dw)
    _check((_lib or load()).pspo_gated_ffn_bwd(
        dy.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), _ptr(preact), N, d, f,
        kind, flags, dx.data_ptr(), dw[0].data_ptr(), dw[1].data_ptr(), dw[2].data_ptr(), workspace.data_ptr(),
        workspace.numel(), _stream(device)))
    return dict(dx=dx, dw_gate=dw[0], dw_up=dw[1], dw_down=dw[2], workspace=workspace)
