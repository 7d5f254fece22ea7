"""GPU: the objectives through the LM head against the float64 oracle, every entry of every output, with the bounds
of tests/objective_util.py."""
import numpy as np
import pytest
import torch

import objective_util as ou
from objective_util import BF, F4, Bounds, close, matrices, np64
from oracle import objectives as oo
from paper_2606_29758_amd import objective, pspo

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


def _poisoned(n):
    """A workspace of the size asked for, filled with NaN."""
    return torch.full((max(n, 256) // 4,), NAN, device="cuda").view(torch.uint8)


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _mask(r, N, share):
    return r.random(N) < share


def _f32(x):
    return np.asarray(x, dtype=np.float32).astype(np.float64)


def _logp(h, w, target, T):
    lp = oo.log_softmax(np64(h) @ np64(w).T / T)
    return lp[np.arange(len(lp)), np64(target)]


def _gradients(o, ref, b, eG, d_hidden, d_w):
    dh, e_h, dw, e_w = b.gradients(ref["G"], eG, d_hidden.dtype == BF, d_w.dtype == BF)
    close(d_hidden, dh, e_h, "d_hidden")
    close(d_w, dw, e_w, "d_w_head")


def run_policy(N, d, V, seed=0, R=3, kl="k3", coef=0.05, T=1.0, masked=0.2, f32=False, wide=1.0):
    r = np.random.default_rng(seed)
    h, w, target = matrices(N, d, V, seed)
    h = h * wide
    l = _logp(h, w, target, T)
    seq, adv = np.sort(r.integers(0, R, N)), _f32(r.normal(size=R))
    shift = r.normal(size=N) * 0.2
    for edge in (np.log(0.8), np.log(1.3)):   # the clip's border decides nothing here
        shift = np.where(np.abs(shift - edge) < 0.01, edge + 0.02, shift)
    old, refp = _f32(l - shift), _f32(l - 0.3 * r.normal(size=N))
    weight = _f32(r.uniform(0.5, 8, N) * np.where(r.random(N) < 0.1, -1, 1))
    off = _mask(r, N, masked)
    weight[off], old[off], refp[off] = 0, NAN, -INF
    h[torch.from_numpy(off).cuda()] = NAN
    tgt = np64(target).copy()
    tgt[off] = V + 7
    adv[-1] = 0.0 if R > 2 else adv[-1]
    want = oo.policy_loss(np64(h), np64(w), tgt, old, weight, seq, adv, float(np.float32(0.2)), float(np.float32(0.3)),
                          float(np.float32(0.01)), logp_ref=refp, kl_coef=float(np.float32(coef)), kl=kl,
                          temperature=float(np.float32(T)))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(d_hidden=torch.full((N, d), NAN, device="cuda"), d_w_head=torch.full((V, d), NAN, device="cuda")) if f32 else {}
    o = objective.policy_loss(h, w, _dev(tgt, torch.int32), _dev(old, F4), _dev(weight, F4), _dev(seq, torch.int32),
                              _dev(adv, F4), N, 0.2, 0.3, 0.01, logp_ref=_dev(refp, F4), kl_coef=coef, kl=kl,
                              temperature=T, err_flag=err,
                              workspace=_poisoned(objective.policy_loss_workspace_bytes(N, d, V)), **kw)
    b = Bounds(np64(h), np64(w), want["on"], want["lp"], T)
    eG, e_loss, e_l = ou.policy_bound(b, want, tgt, old, refp, weight, adv[seq], 0.01, coef, kl)
    close(o["logp_new"], want["logp"], np.where(want["on"], e_l, 0), "logp")
    close(o["loss"], [want["loss"]], e_loss + 1e-12 * abs(want["loss"]), "loss")
    s = np64(o["stats"])
    assert s[2] == want["stats"][2] and s[3] == want["stats"][3] and int(err) == 0
    _gradients(o, want, b, eG, o["d_hidden"], o["d_w_head"])
    return o


def run_preference(N, d, V, seed=0, R=4, P=5, kind="sigmoid", smoothing=0.0, average=False, beta=0.1, T=1.0, masked=0.2,
                   f32=False, ref=True, weights=True, wide=1.0):
    r = np.random.default_rng(seed)
    h, w, target = matrices(N, d, V, seed)
    h = h * wide
    refp = _f32(_logp(h, w, target, T) - 0.05 - 0.2 * r.normal(size=N)) if ref else None
    weight = _f32(r.uniform(0.5, 2, N)) if weights else None
    off = _mask(r, N, masked) if weights else np.zeros(N, dtype=bool)
    tgt = np64(target).copy()
    if weights:
        weight[off], tgt[off] = 0, -100
        h[torch.from_numpy(off).cuda()] = NAN
        if ref:
            refp[off] = NAN
    # rows before the first and behind the last sequence, and an empty one
    cu = np.sort(r.integers(0, N + 1, R + 1))
    if R > 1:
        cu[1] = cu[0]
    a, c = r.integers(0, max(R, 1), P), r.integers(0, max(R, 1), P)
    want = oo.preference_loss(np64(h), np64(w), tgt, cu, a, c, float(np.float32(beta)), 0.25, logp_ref=refp, weight=weight,
                              kind=kind, smoothing=float(np.float32(smoothing)), average=average,
                              temperature=float(np.float32(T)))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(d_hidden=torch.full((N, d), NAN, device="cuda"), d_w_head=torch.full((V, d), NAN, device="cuda")) if f32 else {}
    o = objective.preference_loss(h, w, _dev(tgt, torch.int32), _dev(cu, torch.int32), _dev(a, torch.int32),
                                  _dev(c, torch.int32), N, beta, 0.25, logp_ref=None if refp is None else _dev(refp, F4),
                                  weight=None if weight is None else _dev(weight, F4), kind=kind, smoothing=smoothing,
                                  average=average, temperature=T, err_flag=err,
                                  workspace=_poisoned(objective.preference_workspace_bytes(N, d, V, R, P)), **kw)
    b = Bounds(np64(h), np64(w), want["on"], want["lp"], T)
    eG, e_loss, e_l, e_r, e_m = ou.preference_bound(b, want, tgt, a, c, beta, 0.25, kind)
    close(o["logp_new"], want["logp"], np.where(want["on"], e_l, 0), "logp")
    close(o["seq_ratio"], want["ratio"], e_r, "ratio")
    close(o["margin"], want["margin"], e_m, "margin")
    close(o["loss"], [want["loss"]], e_loss, "loss")
    assert int(err) == 0
    _gradients(o, want, b, eG, o["d_hidden"], o["d_w_head"])
    return o


def run_distill(N, d, V, seed=0, k=5, T=1.0, masked=0.2, f32=False, weights=True, repeats=True, wide=1.0):
    r = np.random.default_rng(seed)
    h, w, target = matrices(N, d, V, seed)
    h = h * wide
    ids = r.integers(0, V, (N, k))   # the same id more than once, where V is small
    if not repeats:
        ids = np.stack([r.permutation(V)[:k] for _ in range(N)])
    ids[:, 0] = np64(target)
    t = _f32(3 * r.normal(size=(N, k)))
    hole = r.random((N, k)) < 0.2
    ids[hole], t[hole] = -1 - r.integers(0, 5, hole.sum()), NAN
    none = (r.random((N, k)) < 0.1) & ~hole
    t[none] = -INF
    ids[none & (r.random((N, k)) < 0.5)] = V + 3     # not an entry, so no invalid id
    empty = r.random(N) < 0.1
    ids[empty] = -1
    weight = _f32(r.uniform(0.5, 8, N)) if weights else None
    off = _mask(r, N, masked) if weights else np.zeros(N, dtype=bool)
    if weights:
        weight[off], ids[off], t[off] = 0, V + 1, INF
        h[torch.from_numpy(off | empty).cuda()] = NAN
    want = oo.distill_loss(np64(h), np64(w), ids, t, float(np.float32(0.01)), weight=weight, temperature=float(np.float32(T)))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(d_hidden=torch.full((N, d), NAN, device="cuda"), d_w_head=torch.full((V, d), NAN, device="cuda")) if f32 else {}
    o = objective.distill_loss(h, w, _dev(ids, torch.int32), _dev(t, F4), N, 0.01,
                               weight=None if weight is None else _dev(weight, F4), temperature=T, err_flag=err,
                               workspace=_poisoned(objective.distill_workspace_bytes(N, d, V, k)), **kw)
    b = Bounds(np64(h), np64(w), want["on"], want["lp"], T)
    eG, e_loss, e_kl = ou.distill_bound(b, want, 0.01)
    close(o["kl"], want["kl"], e_kl, "kl")
    close(o["loss"], [want["loss"]], e_loss, "loss")
    assert int(err) == 0
    _gradients(o, want, b, eG, o["d_hidden"], o["d_w_head"])
    return o


SIZES = [(1, 8, 1), (1, 64, 2), (1, 200, 4099), (2, 8, 7), (3, 64, 64), (16, 128, 65), (17, 200, 255), (33, 72, 2048),
         (63, 136, 2049), (64, 64, 2050), (65, 8, 9), (65, 64, 1000), (127, 520, 257), (129, 64, 4099), (257, 264, 512),
         (300, 72, 130), (513, 64, 2113), (1025, 40, 321),
         # every width that the single pass is built for, its widest and past it, 1 to 4 work-groups of 16 rows
         (5, 256, 60), (9, 392, 70), (20, 520, 333), (16, 1032, 100), (33, 1544, 45), (50, 2056, 40), (12, 2568, 90),
         (40, 3080, 33), (64, 3584, 50), (17, 3584, 1000), (3, 3592, 33), (40, 3600, 70),
         # tiles split along K, 256 x 256 tiles, rows by waves
         (70, 2048, 300), (300, 1024, 700), (2100, 72, 6000), (2300, 136, 515), (4200, 16, 90)]


@pytest.mark.parametrize("N,d,V", SIZES)
def test_policy_sizes(N, d, V):
    run_policy(N, d, V, seed=N + d + V, kl=("k1", "k2", "k3")[(N + d + V) % 3], T=(1.0, 0.7, 2.5)[V % 3], f32=N % 2 == 0)


@pytest.mark.parametrize("N,d,V", SIZES)
def test_preference_sizes(N, d, V):
    kind = ("sigmoid", "squared")[V % 2]
    run_preference(N, d, V, seed=N + d + V, kind=kind, smoothing=0.1 if kind == "sigmoid" else 0.0, average=N % 3 == 0,
                   T=(1.0, 0.7, 2.5)[V % 3], f32=N % 2 == 0)


@pytest.mark.parametrize("N,d,V", SIZES)
def test_distill_sizes(N, d, V):
    run_distill(N, d, V, seed=N + d + V, k=(1, 2, 5, 16, 33, 64)[(N + V) % 6], T=(1.0, 0.7, 2.5)[V % 3], f32=N % 2 == 0)


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("coef", [0.0, 0.3, -0.1])
def test_policy_penalties(kl, coef):
    run_policy(150, 64, 500, seed=5, kl=kl, coef=coef, R=7)


@pytest.mark.parametrize("kw", [dict(R=0, P=0), dict(R=1, P=0), dict(R=1, P=3), dict(R=40, P=500), dict(R=300, P=2),
                                dict(ref=False), dict(weights=False), dict(average=True, kind="squared", beta=2.0),
                                dict(smoothing=1.0), dict(beta=30.0)])
def test_preference_pairs(kw):
    run_preference(**dict(dict(N=150, d=64, V=500, seed=6), **kw))


@pytest.mark.parametrize("kw", [dict(k=64), dict(k=1), dict(weights=False), dict(V=3, k=9), dict(k=40, repeats=False)])
def test_distill_lists(kw):
    run_distill(**dict(dict(N=150, d=64, V=500, seed=8), **kw))


@pytest.mark.parametrize("N,d,T", [(5, 64, 1.0), (40, 64, 1.0), (20, 3592, 1.0), (150, 64, 1.0), (150, 64, 0.25),
                                   (300, 64, 0.05), (2050, 64, 0.25)])
def test_targets_far_below_the_largest_logit(N, d, T):
    """Logits of some hundred times the temperature: groups of entries that pass their row's reference, down to
    rows whose target has no weight left."""
    run_policy(N, d, 1000, seed=1, wide=30.0, T=T, kl="k1")
    run_preference(N, d, 1000, seed=2, wide=30.0, T=T, beta=0.01)
    run_distill(N, d, 1000, seed=3, wide=30.0, T=T, k=3)


@pytest.mark.parametrize("N", [20, 200])
def test_everything_masked(N):
    """No row takes part: zeros, whatever the rows hold."""
    for o in (run_policy(N, 64, 300, masked=1.1), run_preference(N, 64, 300, masked=1.1),
              run_distill(N, 64, 300, masked=1.1)):
        assert not o["d_hidden"].any() and not o["d_w_head"].any()


@pytest.mark.parametrize("N", [5, 40, 150, 2100])
def test_entries_below_the_normal_numbers(N):
    """A row whose largest entry set apart is exp(-100): p is 1 and q is 1 at the first id (logit 0, the others' at most
    -100), q is exp(-1000) = 0 at the second.  Every factor is at most 1 and every |w| at most 120, so no gradient passes
    V 120 (exp(-100) + exp(-100)) < 1e-38."""
    V, d = 40, 8
    w = torch.zeros(V, d, dtype=BF, device="cuda")
    w[1, 0], w[2:, 0] = -100, -120
    h = torch.zeros(N, d, dtype=BF, device="cuda")
    h[:, 0] = 1
    ids = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").repeat(N, 1)
    t = torch.tensor([[0.0, -1000.0]], device="cuda").repeat(N, 1)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = objective.distill_loss(h, w, ids, t, N, 1.0 / N, err_flag=err)
    assert int(err) == 0 and float(o["loss"]) == 0 and bool((o["kl"] == 0).all())
    for g in (o["d_hidden"], o["d_w_head"]):
        assert bool((g.abs() < 1e-37).all())   # (a NaN is not)
