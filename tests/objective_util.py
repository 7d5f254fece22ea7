"""Inputs of the objectives' GPU tests and entry-wise bounds on what the calls may differ from the oracle by.

u = 2^-24 is one float32 rounding, B = 2^-8 half a bf16 step.  Carried through the formulas:
  z     a float32 sum of d exact products: (d + 2) u times the sum of their sizes;
  lse   the mean of z's errors under p, and 64 u + 8 u |z| spread for the exponentials (the instruction's argument
        carries two roundings of up to its size, its result one) and the sums of up to 64 + 8 terms
        of a group (the groups' sums are joined in float64, their scalings take 4 u);
  l     z's and lse's;
  G     B for the softmax entry, B for the factor that makes a row's largest entry set apart exact, the exponent's
        error, and the factor's; an entry set apart its own error and B;
  dH    float32 sums of V terms, dW float32 sums of N terms whose hidden rows, times their factors, take B as well;
        B once more where the output is bf16.
Second-order terms are covered by a factor 1.02 on the whole.
"""
import numpy as np
import torch

from oracle import objectives as oo

U, B = 2.0 ** -24, 2.0 ** -8
BF, F4 = torch.bfloat16, torch.float32


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def matrices(N, d, V, seed, peak=6.0, cap=None):
    """hidden [cap, d], w [V, d] (bf16) and targets whose logits range up to `peak` above the others' sum."""
    g = torch.Generator("cuda").manual_seed(seed)
    cap = N if cap is None else cap
    w = (torch.randn(V, d, device="cuda", generator=g) * (1.2 / d ** 0.5)).to(BF)
    target = torch.randint(0, V, (cap,), device="cuda", generator=g).to(torch.int32)
    up = w[target.long()].float()
    top = (np.log(V) + peak) * torch.rand(cap, 1, device="cuda", generator=g)
    h = torch.randn(cap, d, device="cuda", generator=g) + up * top / up.square().sum(1, keepdim=True).clamp_min(1e-3)
    return h.to(BF), w, target


class Bounds:
    def __init__(self, h, w, on, lp, temperature):
        """h, w, lp: float64; rows that are not `on` count as zeros."""
        s = 1 / temperature
        self.s, self.h, self.w, self.on = s, np.where(on[:, None], h, 0), w, on
        d = h.shape[1]
        self.p, self.lp = np.exp(lp), lp
        self.ez = s * (d + 2) * U * (np.abs(self.h) @ np.abs(w).T)
        spread = lp.max(1, keepdims=True) - lp
        self.e_lse = ((self.p * (self.ez + 8 * U * spread)).sum(1) + 64 * U) * 1.02
        self.ep = self.ez + self.e_lse[:, None] + 8 * U * spread + 8 * U   # relative, of p

    def logp(self, target):
        i = np.arange(len(target))
        t = np.where(self.on, target, 0)
        return self.ez[i, t] + self.e_lse + U * np.abs(self.lp[i, t])

    def of_G(self, G, a, e_a, set_apart, e_set):
        """G's bound: a the factor of p with error e_a ([N]); entries set apart ([N, V] mask) with error e_set."""
        e = np.abs(a)[:, None] * self.p * (2 * B + B * B + self.ep + 6 * U) + e_a[:, None] * self.p
        return np.where(set_apart, e_set + B * (np.abs(G) + e_set), e) * 1.02

    def gradients(self, G, eG, bf16_h, bf16_w):
        (N, V), aw, ah = G.shape, np.abs(self.w), np.abs(self.h)
        dh, dw = oo.gradients(G, self.h, self.w, self.on)
        size = np.abs(G) + eG
        e_h = eG @ aw + (V + 66) * U * (size @ aw)
        e_w = (eG + B * size).T @ ah + (N + 66) * U * (1 + B) * (size.T @ ah)
        if bf16_h:
            e_h = e_h + B * (np.abs(dh) + e_h)
        if bf16_w:
            e_w = e_w + B * (np.abs(dw) + e_w)
        return dh, e_h, dw, e_w


def close(got, want, err, what):
    got = np64(got) if isinstance(got, torch.Tensor) else np.asarray(got)
    assert got.shape == np.shape(want), (what, got.shape, np.shape(want))
    bad = np.isnan(want)
    assert np.array_equal(np.isnan(got), bad), what
    e, tol = np.abs(got - want)[~bad], (np.broadcast_to(err, got.shape) + 1e-30)[~bad]
    assert (e <= tol).all(), (what, float((e / tol).max()))


def through_target(b, o, target, e_delta):
    """G's bound of a loss in the targets' log-probs."""
    N, V = o["G"].shape
    e_l = b.logp(target)
    apart = np.zeros((N, V), dtype=bool)
    i = np.nonzero(b.on & (o["delta"] != 0))[0]
    apart[i, target[i]] = True
    d, l = np.abs(o["delta"]), np.where(b.on, np.nan_to_num(o["logp"]), 0.0)
    e_set = b.s * (e_delta * np.abs(np.expm1(l)) + d * (np.exp(l) * e_l + 4 * U * np.abs(np.expm1(l))))
    return b.of_G(o["G"], b.s * d, b.s * (e_delta + 2 * U * d), apart, e_set[:, None]), e_l


def policy_bound(b, o, target, old, ref, weight, A, scale, coef, kl):
    """Bounds of G, the loss and the log-probs."""
    e_l = b.logp(target)
    l = np.where(b.on, np.nan_to_num(o["logp"]), 0.0)
    c = np.abs(np.where(b.on, weight, 0) * scale)
    rho = np.where(b.on, np.exp(l - np.where(b.on, old, 0)), 0)
    u = l - np.where(b.on, ref, 0)
    curve = {"k1": 0 * u, "k2": 1 + 0 * u, "k3": np.exp(-u)}[kl]
    slope, size = np.abs(oo.kl_slope(u, kl)), np.abs(oo.kl_value(u, kl))
    e_delta = c * 1.02 * (rho * np.abs(A) * (e_l + 8 * U) + abs(coef) * (curve * e_l + 8 * U * slope))
    e_loss = (c * 1.02 * (rho * np.abs(A) * (e_l + 8 * U) + abs(coef) * (slope * e_l + 8 * U * size))).sum()
    eG, _ = through_target(b, o, target, e_delta)
    return eG, e_loss, e_l


def preference_bound(b, o, target, chosen, rejected, beta, scale, kind):
    """Bounds of G, the loss, the log-probs, the ratios and the margins."""
    e_l = b.logp(target)
    R = len(o["ratio"])
    c = np.where(b.on, np.abs(o["weight"]), 0)
    e_r = np.array([(c * e_l)[o["seq"] == r].sum() for r in range(R)]) * np.abs(o["norm"])
    e_coef, e_loss, e_m = np.zeros(R), 0.0, np.zeros(len(chosen))
    for q, (x, y) in enumerate(zip(chosen, rejected)):
        if not (0 <= x < R and 0 <= y < R):
            continue
        e_u = e_r[x] + e_r[y]
        u = o["ratio"][x] - o["ratio"][y]
        e_m[q] = beta * e_u + U * abs(beta * u)
        if kind == "sigmoid":   # |loss'| <= beta, |loss''| <= beta^2 / 4
            e_loss += scale * beta * e_u
            e_du = scale * beta * beta / 4 * e_u
        else:
            e_loss += scale * (2 * abs(u - 1 / (2 * beta)) + e_u) * e_u
            e_du = scale * 2 * e_u
        e_coef[x] += e_du
        e_coef[y] += e_du
    seq = np.where(o["seq"] >= 0, o["seq"], 0)
    e_delta = (e_coef * np.abs(o["norm"]))[seq] * c if R else np.zeros(len(c))
    eG, _ = through_target(b, o, target, e_delta * 1.02 + 4 * U * np.abs(o["delta"]))
    return eG, e_loss * 1.02 + 1e-12 * abs(o["loss"]), e_l, e_r * 1.02 + U * np.abs(o["ratio"]), e_m * 1.02


def distill_bound(b, o, scale):
    """Bounds of G, the loss and the rows' divergences."""
    c = np.abs(o["weight"] * scale)
    q = o["q"]
    e_l = b.ez + b.e_lse[:, None]
    kl = np.nan_to_num(o["kl"])
    e_kl = (q * e_l).sum(1) + U * np.abs(kl)
    apart = q > 0
    e_set = (b.s * c)[:, None] * (b.p * (e_l + 4 * U) + 4 * U * (b.p + q))
    eG = b.of_G(o["G"], b.s * c, 2 * U * b.s * c, apart, e_set)
    return eG, (c * e_kl).sum() * 1.02 + 1e-12 * abs(o["loss"]), e_kl * 1.02
