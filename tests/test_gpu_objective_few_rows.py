"""GPU: the head's gradient of up to 64 rows, whose roundings no sum over many rows averages: a row's entry at its target
is exact up to the log-prob's error, and so is its product with the hidden row.

With u = 2^-24 and B = 2^-8: an entry of G at the target is off by its own error (objective_util) and, as two bf16 parts of
f E, by 2^-16 of itself; the others take B for their rounding and B for the factor that makes the target's exact; the
hidden rows go in as they are, the sum of N products is float32.
"""
import numpy as np
import pytest
import torch

import objective_util as ou
from objective_util import F4, Bounds, U, close, matrices, np64
from oracle import objectives as oo
from paper_2606_29758_amd import objective

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,d,V", [(1, 64, 300), (7, 136, 2000), (9, 64, 1000), (16, 1032, 700), (16, 3584, 90), (17, 64, 1000),
                                   (32, 200, 4099), (33, 72, 2048), (48, 1544, 100), (64, 264, 513)])
def test_the_head_gradient_takes_no_rounding_of_the_rows(N, d, V, accumulate):
    r = np.random.default_rng(N)
    h, w, target = matrices(N, d, V, N)
    lp = oo.log_softmax(np64(h) @ np64(w).T)
    tgt = np64(target)
    old = np.float32(lp[np.arange(N), tgt]).astype(np.float64)
    weight, adv = np.float32(r.uniform(0.5, 8, N)).astype(np.float64), np.float32(r.uniform(0.5, 2, 3)).astype(np.float64)
    seq = np.sort(r.integers(0, 3, N))
    dev = lambda a, t=F4: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()   # noqa: E731
    scale = float(np.float32(0.01))
    want = oo.policy_loss(np64(h), np64(w), tgt, old, weight, seq, adv, float(np.float32(0.2)), float(np.float32(0.2)), scale)
    before = torch.full((V, d), 0.0 if accumulate else float("nan"), device="cuda")
    o = objective.policy_loss(h, w, target, dev(old), dev(weight), dev(seq, torch.int32), dev(adv), N, 0.2, 0.2, 0.01,
                              d_w_head=before, accumulate=accumulate)
    b = Bounds(np64(h), np64(w), want["on"], want["lp"], 1.0)
    e_l = b.logp(tgt)
    d_l = np.abs(want["delta"])
    e_delta = d_l * 1.02 * (e_l + 8 * U)
    i = np.arange(N)
    eG = b.p * (d_l * (2 * ou.B + 6 * U) + e_delta)[:, None] + d_l[:, None] * b.p * b.ep
    l = want["logp"]
    eG[i, tgt] = e_delta * np.abs(np.expm1(l)) + d_l * np.exp(l) * e_l + (2.0 ** -16 + 4 * U) * np.abs(want["G"][i, tgt])
    ah = np.abs(np64(h))
    tol = 1.02 * (eG.T @ ah + (N + 4) * U * ((np.abs(want["G"]) + eG).T @ ah))
    close(o["d_w_head"], want["G"].T @ np64(h), tol, "d_w_head")
