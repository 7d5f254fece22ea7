"""Python binding of the objectives through the LM head (include/pspo_objective.h): argument marshalling only.

The clipped policy loss with a penalty on the divergence from a reference policy, a preference loss on pairs
of sequences, and distillation from a teacher's top logits; each call gives the loss and the gradients of the
hidden rows and of the head.  As in ``pspo``: every step runs in the HIP kernels of libpspo.so on the current
stream, tensors must be on the current device, a missing library raises.  All calls take the first N rows of
their per-token tensors.  A row of weight 0 takes no part and nothing else of it is read.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import pspo
from .layer import _F32, _I32, _P, _SZ, _U32, _apart, _check, _count, _exact, _fits, _here, _ints, _ptr, _rows, _stream, _type

DH_F32, DW_F32, PREF_AVERAGE = 2048, 4096, 8192
KL_KINDS = {"k1": 1, "k2": 2, "k3": 3}
PREFERENCES = {"sigmoid": 0, "squared": 1}

_SIGNATURES = {
    "pspo_policy_loss_workspace_bytes": (_SZ, [_I32] * 4),
    "pspo_preference_workspace_bytes": (_SZ, [_I32] * 6),
    "pspo_distill_workspace_bytes": (_SZ, [_I32] * 5),
    "pspo_policy_loss_fwd_bwd": (ctypes.c_int, [_P] * 8 + [_I32] * 4 + [_F32, _F32, _F32, _I32, _F32, _F32, _U32] +
                                 [_P] * 6 + [_P, _SZ, _P]),
    "pspo_preference_fwd_bwd": (ctypes.c_int, [_P] * 8 + [_I32] * 6 + [_F32, _F32, _F32, _F32, _U32] + [_P] * 7 +
                                [_P, _SZ, _P]),
    "pspo_distill_fwd_bwd": (ctypes.c_int, [_P] * 5 + [_I32] * 4 + [_F32, _F32, _U32] + [_P] * 5 + [_P, _SZ, _P]),
}

_lib = None


def load() -> ctypes.CDLL:
    """libpspo.so with the signatures of the objectives; raises if it is missing."""
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


def _name(kinds: dict, kind: str, what: str) -> int:
    if kind not in kinds:
        raise ValueError(f"{what} must be one of {sorted(kinds)}, got {kind!r}")
    return kinds[kind]


def _head(hidden, w_head, N: int):
    """(device, d, V) of the matrices."""
    device = torch.cuda.current_device()
    if not isinstance(w_head, torch.Tensor):
        raise TypeError("w_head must be a torch.Tensor")
    if w_head.dim() != 2:
        raise ValueError("w_head must be [V, d]")
    V, d = w_head.shape
    _fits(max(V, d), "V and d")
    _here(w_head, torch.bfloat16, "w_head", device)
    _rows(hidden, N, (d,), "hidden")
    _here(hidden, torch.bfloat16, "hidden", device)
    return device, d, V


def _floats(t, n: int, name: str, device: int) -> None:
    if t is None:
        return
    _here(t, torch.float32, name, device)
    if t.dim() != 1 or t.shape[0] < n:
        raise ValueError(f"{name} must be [>= {n}], got {list(t.shape)}")


def _needed(**tensors) -> None:
    for name, t in tensors.items():
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")


class _Outputs:
    """The gradients, the workspace and the flags of a call, checked against what it reads."""

    def __init__(self, w_head, N, d, V, device, read, d_hidden, d_w_head, want_hidden, want_head, accumulate, workspace,
                 err_flag, need):
        dev = w_head.device
        if err_flag is not None:
            _here(err_flag, torch.int32, "err_flag", device)
            if err_flag.numel() < 1:
                raise ValueError("err_flag must hold one word")
        if accumulate and d_w_head is None:
            raise ValueError("accumulate needs d_w_head")
        read = (*read, err_flag)
        if d_hidden is not None:
            if not want_hidden:
                raise ValueError("d_hidden is given, but not wanted")
            _type(d_hidden, "d_hidden")
            _rows(d_hidden, N, (d,), "d_hidden")
            _here(d_hidden, d_hidden.dtype, "d_hidden", device)
            _apart(d_hidden, "d_hidden", *read)
        elif want_hidden:
            d_hidden = torch.empty((N, d), dtype=torch.bfloat16, device=dev)
        if d_w_head is not None:
            if not want_head:
                raise ValueError("d_w_head is given, but not wanted")
            _type(d_w_head, "d_w_head")
            _exact(d_w_head, (V, d), "d_w_head")
            _here(d_w_head, d_w_head.dtype, "d_w_head", device)
            _apart(d_w_head, "d_w_head", *read, d_hidden)
        elif want_head:
            d_w_head = torch.empty((V, d), dtype=torch.bfloat16, device=dev)
        if workspace is None:
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        else:
            _here(workspace, torch.uint8, "workspace", device)
            _apart(workspace, "workspace", *read, d_hidden, d_w_head, used=need)
        self.d_hidden, self.d_w_head, self.workspace = d_hidden, d_w_head, workspace
        self.loss = torch.empty(1, dtype=torch.float64, device=dev)
        self.flags = ((DH_F32 if d_hidden is not None and d_hidden.dtype == torch.float32 else 0) |
                      (DW_F32 if d_w_head is not None and d_w_head.dtype == torch.float32 else 0) |
                      (pspo.PSPO_ACCUMULATE_DW if accumulate else 0))
        self.last = (workspace.data_ptr(), workspace.numel(), _stream(device))

    def result(self, N, **more) -> dict:
        dh = self.d_hidden
        if dh is not None and dh.shape[0] != N:
            dh = dh[:N]
        return dict(loss=self.loss, d_hidden=dh, d_w_head=self.d_w_head, workspace=self.workspace, **more)


def policy_loss_workspace_bytes(N: int, d: int, V: int, grads: bool = True) -> int:
    """Bytes of workspace that policy_loss takes for up to N rows."""
    return int(load().pspo_policy_loss_workspace_bytes(_fits(N, "N"), _fits(d, "d"), _fits(V, "V"), int(grads)))


def preference_workspace_bytes(N: int, d: int, V: int, R: int, P: int, grads: bool = True) -> int:
    """Bytes of workspace that preference_loss takes for up to N rows, R sequences and P pairs."""
    return int(load().pspo_preference_workspace_bytes(_fits(N, "N"), _fits(d, "d"), _fits(V, "V"), _fits(R, "R"),
                                                      _fits(P, "P"), int(grads)))


def distill_workspace_bytes(N: int, d: int, V: int, k: int, grads: bool = True) -> int:
    """Bytes of workspace that distill_loss takes for up to N rows and lists of k entries."""
    return int(load().pspo_distill_workspace_bytes(_fits(N, "N"), _fits(d, "d"), _fits(V, "V"), _fits(k, "k"),
                                                   int(grads)))


def policy_loss(hidden, w_head, target, logp_old, weight, seq_id, advantage, N: int, eps_low: float, eps_high: float,
                loss_scale: float, logp_ref: Optional[torch.Tensor] = None, kl_coef: float = 0.0, kl: str = "k3",
                temperature: float = 1.0, d_hidden: Optional[torch.Tensor] = None,
                d_w_head: Optional[torch.Tensor] = None, want_hidden: bool = True, want_head: bool = True,
                accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                err_flag: Optional[torch.Tensor] = None) -> dict:
    """Clipped policy loss + kl_coef * divergence from a reference policy, with its gradients.

    loss = loss_scale sum_i weight_i (kl_coef kl(l_i - logp_ref_i) - min(rho_i A_i, clip(rho_i) A_i)), l_i the
    target's log-prob at `temperature`, rho_i = exp(l_i - logp_old_i); kl: "k1" (u), "k2" (u^2 / 2), "k3"
    (exp(-u) - 1 + u).  hidden: bf16 [>=N, d]; w_head: bf16 [V, d]; target, seq_id: int32, logp_old, logp_ref,
    weight: float32, all [>=N]; advantage: float32 [R].  d_hidden ([>=N, d]) and d_w_head ([V, d]) may be given,
    bf16 or float32; accumulate adds to a float32 d_w_head; want_head=False leaves the head's gradient out.
    Returns loss (float64 [1]), d_hidden, d_w_head (bf16 unless given), logp_new (float32 [N]) and stats
    (float64 [4]: the scaled sums of the clipped gain and of the divergence, the clipped rows, the rows taken).
    """
    N = _count(N)
    kind = _name(KL_KINDS, kl, "kl")
    device, d, V = _head(hidden, w_head, N)
    _needed(target=target, logp_old=logp_old, weight=weight, seq_id=seq_id, advantage=advantage)
    _ints(target, N, "target", device)
    _ints(seq_id, N, "seq_id", device)
    for name, t in (("logp_old", logp_old), ("logp_ref", logp_ref), ("weight", weight)):
        _floats(t, N, name, device)
    _floats(advantage, 0, "advantage", device)
    R = _fits(advantage.shape[0], "R")
    lib = _lib or load()
    need = lib.pspo_policy_loss_workspace_bytes(N, d, V, int(want_hidden or want_head))
    o = _Outputs(w_head, N, d, V, device, (hidden, w_head, target, logp_old, logp_ref, weight, seq_id, advantage),
                 d_hidden, d_w_head, want_hidden, want_head, accumulate, workspace, err_flag, need)
    logp = torch.empty(N, dtype=torch.float32, device=w_head.device)
    stats = torch.empty(4, dtype=torch.float64, device=w_head.device)
    _check(lib.pspo_policy_loss_fwd_bwd(
        hidden.data_ptr(), w_head.data_ptr(), target.data_ptr(), logp_old.data_ptr(), _ptr(logp_ref),
        weight.data_ptr(), seq_id.data_ptr(), advantage.data_ptr(), N, d, V, R, eps_low, eps_high, kl_coef, kind,
        temperature, loss_scale, o.flags, o.loss.data_ptr(), _ptr(o.d_hidden), _ptr(o.d_w_head), logp.data_ptr(),
        stats.data_ptr(), _ptr(err_flag), *o.last))
    return o.result(N, logp_new=logp, stats=stats)


def preference_loss(hidden, w_head, target, cu_seqlens, chosen, rejected, N: int, beta: float, loss_scale: float,
                    logp_ref: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                    kind: str = "sigmoid", smoothing: float = 0.0, average: bool = False, temperature: float = 1.0,
                    d_hidden: Optional[torch.Tensor] = None, d_w_head: Optional[torch.Tensor] = None,
                    want_hidden: bool = True, want_head: bool = True, accumulate: bool = False,
                    workspace: Optional[torch.Tensor] = None, err_flag: Optional[torch.Tensor] = None) -> dict:
    """Preference loss on pairs of sequences, with its gradients.

    ratio_r = sum over the rows of sequence r of weight_i (l_i - logp_ref_i) (average: their weighted mean),
    u = ratio[chosen] - ratio[rejected];  loss = loss_scale times the sum over the pairs of
    -(1 - smoothing) log s(beta u) - smoothing log s(-beta u) ("sigmoid", s the logistic function) or
    (u - 1 / (2 beta))^2 ("squared").  cu_seqlens: int32 [R + 1]; chosen, rejected: int32 [P]; logp_ref (None:
    zeros) and weight (None: ones): float32 [>=N]; the other arguments as in policy_loss.  Rows outside every
    sequence get their log-prob and zero gradient, whatever they hold.
    Returns loss, d_hidden, d_w_head, logp_new [N], seq_ratio [R] and margin [P] (beta u).
    """
    N = _count(N)
    which = _name(PREFERENCES, kind, "kind")
    device, d, V = _head(hidden, w_head, N)
    _needed(target=target, cu_seqlens=cu_seqlens, chosen=chosen, rejected=rejected)
    _ints(target, N, "target", device)
    _ints(cu_seqlens, 1, "cu_seqlens", device)
    _ints(chosen, 0, "chosen", device)
    _ints(rejected, 0, "rejected", device)
    if chosen.shape != rejected.shape:
        raise ValueError(f"chosen and rejected must have one length, got {list(chosen.shape)} and {list(rejected.shape)}")
    for name, t in (("logp_ref", logp_ref), ("weight", weight)):
        _floats(t, N, name, device)
    R, P = _fits(cu_seqlens.shape[0] - 1, "R"), _fits(chosen.shape[0], "P")
    lib = _lib or load()
    need = lib.pspo_preference_workspace_bytes(N, d, V, R, P, int(want_hidden or want_head))
    o = _Outputs(w_head, N, d, V, device, (hidden, w_head, target, cu_seqlens, chosen, rejected, logp_ref, weight),
                 d_hidden, d_w_head, want_hidden, want_head, accumulate, workspace, err_flag, need)
    logp, ratio, margin = (torch.empty(n, dtype=torch.float32, device=w_head.device) for n in (N, R, P))
    flags = o.flags | (PREF_AVERAGE if average else 0)
    _check(lib.pspo_preference_fwd_bwd(
        hidden.data_ptr(), w_head.data_ptr(), target.data_ptr(), _ptr(logp_ref), _ptr(weight), cu_seqlens.data_ptr(),
        chosen.data_ptr(), rejected.data_ptr(), N, d, V, R, P, which, beta, smoothing, temperature, loss_scale, flags,
        o.loss.data_ptr(), _ptr(o.d_hidden), _ptr(o.d_w_head), logp.data_ptr(), ratio.data_ptr(), margin.data_ptr(),
        _ptr(err_flag), *o.last))
    return o.result(N, logp_new=logp, seq_ratio=ratio, margin=margin)


def distill_loss(hidden, w_head, topk_ids, topk_logit, N: int, loss_scale: float,
                 weight: Optional[torch.Tensor] = None, temperature: float = 1.0,
                 d_hidden: Optional[torch.Tensor] = None, d_w_head: Optional[torch.Tensor] = None,
                 want_hidden: bool = True, want_head: bool = True, accumulate: bool = False,
                 workspace: Optional[torch.Tensor] = None, err_flag: Optional[torch.Tensor] = None) -> dict:
    """Divergence of the policy from a teacher known through its top logits (or log-probs), with its gradients.

    loss = loss_scale sum_i weight_i kl_i, kl_i = sum_j q_ij (log q_ij - log p_i(id_ij)), q_i the softmax of
    topk_logit[i] / temperature over the list, p_i the policy at `temperature` over the whole vocabulary.
    topk_ids: int32 [>=N, k] (negative: no entry), topk_logit: float32 [>=N, k] (-inf: none either), k <= 64;
    weight: float32 [>=N] (None: ones); the other arguments as in policy_loss.
    Returns loss, d_hidden, d_w_head and kl (float32 [N]).
    """
    N = _count(N)
    device, d, V = _head(hidden, w_head, N)
    _needed(topk_ids=topk_ids, topk_logit=topk_logit)
    if topk_ids.dim() != 2:
        raise ValueError("topk_ids must be [>= N, k]")
    k = _fits(topk_ids.shape[1], "k")
    _rows(topk_ids, N, (k,), "topk_ids")
    _rows(topk_logit, N, (k,), "topk_logit")
    _here(topk_ids, torch.int32, "topk_ids", device)
    _here(topk_logit, torch.float32, "topk_logit", device)
    _floats(weight, N, "weight", device)
    lib = _lib or load()
    need = lib.pspo_distill_workspace_bytes(N, d, V, k, int(want_hidden or want_head))
    o = _Outputs(w_head, N, d, V, device, (hidden, w_head, topk_ids, topk_logit, weight), d_hidden, d_w_head,
                 want_hidden, want_head, accumulate, workspace, err_flag, need)
    kl = torch.empty(N, dtype=torch.float32, device=w_head.device)
    _check(lib.pspo_distill_fwd_bwd(
        hidden.data_ptr(), w_head.data_ptr(), topk_ids.data_ptr(), topk_logit.data_ptr(), _ptr(weight), N, d, V, k,
        temperature, loss_scale, o.flags, o.loss.data_ptr(), _ptr(o.d_hidden), _ptr(o.d_w_head), kl.data_ptr(),
        _ptr(err_flag), *o.last))
    return o.result(N, kl=kl)
