"""Float64 oracle of the objectives through the LM head: policy loss with a reference penalty, preference
pairs, distillation from top logits.

Written from the formulas, numpy only; shares no code with the library.  bf16 and float32 inputs are given as the
float64 values they stand for.  Every function returns the loss, the per-row quantity and the dense logit gradient
G [N, V] = d loss / d (h W^T), from which d_hidden = G W and d_w = G^T h follow.
"""
import numpy as np


def log_softmax(z):
    m = z.max(axis=1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))


def _rows(weight, N):
    w = np.ones(N) if weight is None else np.asarray(weight, dtype=np.float64)
    return w, w != 0


def _through(delta, lp, target, on, inv_t):
    """G of d loss / d log p(target) = delta."""
    G = -delta[:, None] * np.exp(lp) * inv_t
    i = np.nonzero(on)[0]
    G[i, target[i]] = -delta[i] * np.expm1(lp[i, target[i]]) * inv_t
    G[~on] = 0
    return G


def gradients(G, hidden, w, on):
    h = np.where(on[:, None], hidden, 0)
    return G @ w, G.T @ h


def _logits(hidden, w, on, inv_t):
    return np.where(on[:, None], hidden, 0) @ w.T * inv_t


def kl_value(u, kind):
    return {"k1": lambda: u, "k2": lambda: u * u / 2, "k3": lambda: np.expm1(-u) + u}[kind]()


def kl_slope(u, kind):
    return {"k1": lambda: np.ones_like(u), "k2": lambda: u, "k3": lambda: -np.expm1(-u)}[kind]()


def policy_loss(hidden, w, target, logp_old, weight, seq_id, advantage, eps_low, eps_high, scale, logp_ref=None,
                kl_coef=0.0, kl="k3", temperature=1.0):
    N, V = hidden.shape[0], w.shape[0]
    c, on = _rows(weight, N)
    bad = on & ((target < 0) | (target >= V) | (seq_id < 0) | (seq_id >= len(advantage)))
    on = on & ~bad
    lp = log_softmax(_logits(hidden, w, on, 1 / temperature))
    i = np.nonzero(on)[0]
    l = lp[i, target[i]]
    A = advantage[seq_id[i]]
    rho = np.exp(l - logp_old[i])
    gain = np.minimum(rho * A, np.clip(rho, 1 - eps_low, 1 + eps_high) * A)
    passes = ((A > 0) & (rho <= 1 + eps_high)) | ((A < 0) & (rho >= 1 - eps_low))
    d = -np.where(passes, rho * A, 0.0)
    div = np.zeros_like(l)
    if logp_ref is not None:
        u = l - logp_ref[i]
        div = kl_value(u, kl)
        if kl_coef:
            d = d + kl_coef * kl_slope(u, kl)
    delta = np.zeros(N)
    delta[i] = scale * c[i] * d
    logp = np.where(bad, np.nan, 0.0)
    logp[i] = l
    gains, divs = scale * (c[i] * gain).sum(), scale * (c[i] * div).sum()
    return dict(loss=(kl_coef * divs if kl_coef else 0.0) - gains, logp=logp, on=on, delta=delta, lp=lp,
                G=_through(delta, lp, target, on, 1 / temperature),
                stats=np.array([gains, divs, ((A != 0) & ~passes).sum(), on.sum()], dtype=np.float64))


def preference_loss(hidden, w, target, cu, chosen, rejected, beta, scale, logp_ref=None, weight=None, kind="sigmoid",
                    smoothing=0.0, average=False, temperature=1.0):
    N, V = hidden.shape[0], w.shape[0]
    R = len(cu) - 1
    c, on = _rows(weight, N)
    bad = on & ((target < 0) | (target >= V))
    on = on & ~bad
    lp = log_softmax(_logits(hidden, w, on, 1 / temperature))
    logp = np.where(bad, np.nan, 0.0)
    i = np.nonzero(on)[0]
    logp[i] = lp[i, target[i]]
    ratio, norm = np.zeros(R), np.ones(R)
    seq = np.full(N, -1)
    for r in range(R):
        at = np.arange(min(max(cu[r], 0), N), min(max(cu[r + 1], 0), N))
        seq[at] = r
        at = at[on[at]]
        ratio[r] = (c[at] * (logp[at] - (0 if logp_ref is None else logp_ref[at]))).sum()
        if average:
            norm[r] = 1 / c[at].sum() if c[at].sum() else 0.0
    ratio = ratio * norm
    coef, loss, margin = np.zeros(R), 0.0, np.full(len(chosen), np.nan)
    for q, (a, b) in enumerate(zip(chosen, rejected)):
        if not (0 <= a < R and 0 <= b < R):
            continue
        u = ratio[a] - ratio[b]
        x = beta * u
        margin[q] = x
        if kind == "sigmoid":
            loss += (1 - smoothing) * np.logaddexp(0, -x) + smoothing * np.logaddexp(0, x)
            du = beta * (smoothing * np.exp(-np.logaddexp(0, -x)) - (1 - smoothing) * np.exp(-np.logaddexp(0, x)))
        else:
            loss += (u - 1 / (2 * beta)) ** 2
            du = 2 * (u - 1 / (2 * beta))
        coef[a] += scale * du
        coef[b] -= scale * du
    in_seq = on & (seq >= 0)
    delta = np.zeros(N)
    delta[in_seq] = (coef * norm)[seq[in_seq]] * c[in_seq]
    return dict(loss=scale * loss, logp=logp, on=on, delta=delta, lp=lp, seq=seq, ratio=ratio, margin=margin, norm=norm,
                weight=c, G=_through(delta, lp, target, in_seq, 1 / temperature))


def distill_loss(hidden, w, ids, teacher, scale, weight=None, temperature=1.0):
    N, V = hidden.shape[0], w.shape[0]
    c, on = _rows(weight, N)
    there = (ids >= 0) & ~(np.where(ids >= 0, teacher, 0) == -np.inf)
    bad = on & (there & (ids >= V)).any(1)
    on = on & there.any(1) & ~bad
    inv_t = 1 / temperature
    lp = log_softmax(_logits(hidden, w, on, inv_t))
    kl = np.where(bad, np.nan, 0.0)
    G = np.zeros((N, V))
    q_all = np.zeros((N, V))
    for i in np.nonzero(on)[0]:
        j = np.nonzero(there[i])[0]
        t = teacher[i, j] * inv_t
        e = np.exp(t - t.max())
        np.add.at(q_all[i], ids[i, j], e / e.sum())
        v = np.nonzero(q_all[i])[0]
        q = q_all[i, v]
        kl[i] = (q * (np.log(q) - lp[i, v])).sum()
        G[i] = scale * c[i] * inv_t * (np.exp(lp[i]) - q_all[i])
    return dict(loss=(scale * c[on] * kl[on]).sum(), kl=kl, on=on, lp=lp, q=q_all, G=G, weight=np.where(on, c, 0))
