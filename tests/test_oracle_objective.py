"""Pins of the objectives' oracle: its gradients against differences of its own losses, and what the formulas say
of simple inputs."""
import numpy as np
import pytest

from oracle import objectives as oo


def _inputs(seed, N=9, d=5, V=13):
    r = np.random.default_rng(seed)
    return dict(h=r.normal(size=(N, d)), w=r.normal(size=(V, d)), target=r.integers(0, V, N),
                weight=r.uniform(0.5, 3, N) * (np.arange(N) != 4), ref=r.normal(size=N) - 2, r=r)


def _policy(x, h, w, **kw):
    r = np.random.default_rng(7)
    N = h.shape[0]
    seq, adv = np.sort(r.integers(0, 3, N)), np.array([1.3, -0.7, 0.4])
    return oo.policy_loss(h, w, x["target"], x["old"], x["weight"], seq, adv, 0.2, 0.3, 0.25, logp_ref=x["ref"], **kw)


def _calls(x):
    cu = np.array([0, 2, 2, 6, 9])
    chosen, rejected = np.array([0, 2, 2, 3]), np.array([2, 3, 0, 3])
    ids = np.array([[1, 5, 1, -1]] * 9)
    t = np.random.default_rng(3).normal(size=ids.shape)
    t[:, 3] = np.nan
    for kl in ("k1", "k2", "k3"):
        yield lambda h, w, kl=kl: _policy(x, h, w, kl=kl, kl_coef=0.3, temperature=0.7)
    for kind, sm in (("sigmoid", 0.0), ("sigmoid", 0.2), ("squared", 0.0)):
        for avg in (False, True):
            yield lambda h, w, kind=kind, sm=sm, avg=avg: oo.preference_loss(
                h, w, x["target"], cu, chosen, rejected, 0.4, 0.5, logp_ref=x["ref"], weight=x["weight"], kind=kind,
                smoothing=sm, average=avg, temperature=1.4)
    yield lambda h, w: oo.distill_loss(h, w, ids, t, 0.5, weight=x["weight"], temperature=1.7)


@pytest.mark.parametrize("seed", range(3))
def test_gradients_are_those_of_the_loss(seed):
    x = _inputs(seed)
    lp = oo.log_softmax(x["h"] @ x["w"].T / 0.7)
    x["old"] = lp[np.arange(9), x["target"]] - np.array([0.1, -0.1, 0.5, -0.5, 0.05, 0.3, -0.4, 0.02, -0.05])
    for call in _calls(x):
        o = call(x["h"], x["w"])
        dh, dw = oo.gradients(o["G"], x["h"], x["w"], o["on"])
        for name, at, g in (("h", x["h"], dh), ("w", x["w"], dw)):
            for _ in range(6):
                i, j = x["r"].integers(at.shape[0]), x["r"].integers(at.shape[1])
                e = np.zeros_like(at)
                e[i, j] = 1e-5
                args = [(at + s * e, x["w"]) if name == "h" else (x["h"], at + s * e) for s in (1, -1)]
                diff = (call(*args[0])["loss"] - call(*args[1])["loss"]) / 2e-5
                # central differences over 1e-5: truncation (1e-5)^2 / 6 times a third derivative, which for the
                # steepest of these losses, exp(-log p) with |entries| <= 3 at temperature 0.7, is (2 * 3 / 0.7)^3 =
                # 630 times the loss: 1.1e-8 of it (k3 far below its reference: a loss of 5e5); rounding a few
                # 2^-53 / 1e-5 = 1e-11 of it
                tol = 1e-6 * (1 + abs(g[i, j])) + 1.2e-8 * abs(call(x["h"], x["w"])["loss"])
                assert abs(diff - g[i, j]) <= tol, (name, i, j, diff, g[i, j])


def test_rows_left_out_are_not_read():
    x = _inputs(0)
    x["old"] = x["ref"] * 1.0
    h = x["h"].copy()
    h[4] = np.nan
    for a, b in zip(_calls(x), _calls(x)):
        o, p = a(x["h"], x["w"]), b(h, x["w"])
        assert o["loss"] == p["loss"] and np.array_equal(o["G"], p["G"]) and not o["G"][4].any()


def test_simple_values():
    x = _inputs(1)
    z = np.zeros((9, 5))
    # a flat policy and a flat teacher over all ids: no divergence, no gradient
    o = oo.distill_loss(z, x["w"], np.arange(13)[None].repeat(9, 0), np.zeros((9, 13)), 1.0)
    assert np.allclose(o["kl"], 0, atol=1e-12) and np.allclose(o["G"], 0, atol=1e-12)
    # one id holds all of the teacher: its negative log-prob
    o = oo.distill_loss(z, x["w"], np.full((9, 2), 3), np.zeros((9, 2)), 1.0)
    assert np.allclose(o["kl"], np.log(13)) and np.allclose(o["G"].sum(1), 0)
    # a policy equal to its reference: log 2 a pair, whatever beta
    lp = oo.log_softmax(x["h"] @ x["w"].T)[np.arange(9), x["target"]]
    o = oo.preference_loss(x["h"], x["w"], x["target"], [0, 4, 9], [0], [1], 0.3, 1.0, logp_ref=lp)
    assert np.isclose(o["loss"], np.log(2)) and np.allclose(o["ratio"], 0)
    # a pair of one sequence with itself moves nothing
    o = oo.preference_loss(x["h"], x["w"], x["target"], [0, 4, 9], [1], [1], 0.3, 1.0)
    assert not o["G"].any()
    # the policy at its old log-probs, no penalty: -sum of weighted advantages
    c, A = x["weight"], np.array([0.5, -1.0])
    seq = np.array([0] * 4 + [1] * 5)
    o = oo.policy_loss(x["h"], x["w"], x["target"], lp, c, seq, A, 0.2, 0.2, 1.0)
    assert np.isclose(o["loss"], -(c * A[seq]).sum())
