"""Float64 oracle of the layer operators: head norms with rotation, dropout, gated feed-forward.

Written from the formulas, numpy only; shares no code with the library.  bf16 inputs are given as
the float64 values they stand for.
"""
import numpy as np

from .philox import philox4x32


# ---------------------------------------------------------------------------
# norms of queries and keys with the position rotation
# ---------------------------------------------------------------------------

def positions(seq_id, cu_seqlens, first_pos, N):
    """pos_n = first_pos[r] + n - cu[r]; 0 where r is out of range."""
    out = np.zeros(N, dtype=np.int64)
    R = len(cu_seqlens) - 1
    for n in range(N):
        r = int(seq_id[n])
        if 0 <= r < R:
            out[n] = (0 if first_pos is None else int(first_pos[r])) + n - int(cu_seqlens[r])
    return out


def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(z, pos, inv_freq, interleaved, back=False):
    """z: [N, H, D]; the first 2 len(inv_freq) entries turned by pos * inv_freq (back: the transpose)."""
    rot = 2 * len(inv_freq)
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * np.asarray(inv_freq, dtype=np.float64)[None, None]
    c, s = np.cos(ang), np.sin(ang) * (-1.0 if back else 1.0)
    a, b = _pairs(rot, interleaved)
    out = np.array(z, dtype=np.float64)
    out[..., a] = z[..., a] * c - z[..., b] * s
    out[..., b] = z[..., a] * s + z[..., b] * c
    return out


def qk_norm_rope(x, w, pos, inv_freq, eps, interleaved=False, norm=True):
    """One side (queries or keys): x [N, H, D], w [D] or None."""
    z = x
    if norm:
        z = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        if w is not None:
            z = z * w
    return rotate(z, pos, inv_freq, interleaved)


def qk_norm_rope_bwd(dout, x, w, pos, inv_freq, eps, interleaved=False, norm=True):
    """dx [N, H, D] and dw [D] (None without a norm)."""
    dz = rotate(dout, pos, inv_freq, interleaved, back=True)
    if not norm:
        return dz, None
    rstd = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    xhat = x * rstd
    dw = (dz * xhat).sum(axis=(0, 1))
    dzw = dz if w is None else dz * w
    return rstd * (dzw - xhat * np.mean(dzw * xhat, axis=-1, keepdims=True)), dw


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

def keep_threshold(p):
    return min(max(int(np.floor((1.0 - p) * 65536.0 + 0.5)), 1), 65536)


def dropout_mask(rows, d, p, seed, offset):
    """bool [len(rows), d]: kept entries."""
    T = keep_threshold(p)
    key = (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    out = np.zeros((len(rows), d), dtype=bool)
    for n, row in enumerate(rows):
        for g in range(d // 8):
            words = philox4x32((int(row) & 0xFFFFFFFF, g + 1, offset & 0xFFFFFFFF, (offset >> 32) & 0xFFFFFFFF), key)
            for i in range(8):
                out[n, 8 * g + i] = ((words[i // 2] >> (16 * (i % 2))) & 0xFFFF) < T
    return out


def dropout_add(x, residual, mask, p):
    y = np.where(mask, np.where(mask, x, 0.0) * (65536.0 / keep_threshold(p)), 0.0)
    return y if residual is None else residual + y


# ---------------------------------------------------------------------------
# gated feed-forward block
# ---------------------------------------------------------------------------

def activation(g, act):
    """act(g) and act'(g)."""
    if act == "silu":
        s = np.where(g >= 0, 1.0, np.exp(-np.abs(g))) / (1.0 + np.exp(-np.abs(g)))
        return g * s, s * (1.0 + g * (1.0 - s))
    a = np.sqrt(2.0 / np.pi)
    t = np.tanh(a * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 0.134145 * g * g)


def gated_ffn(x, wg, wu, wd, act):
    """y [N, d] and the pre-activations [N, 2 f] (gate, up)."""
    g, u = x @ wg.T, x @ wu.T
    return (activation(g, act)[0] * u) @ wd.T, np.concatenate([g, u], axis=1)


def gated_ffn_bwd(dy, x, wg, wu, wd, act):
    """dx, dwg, dwu, dwd."""
    g, u = x @ wg.T, x @ wu.T
    a, da = activation(g, act)
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ (a * u)
