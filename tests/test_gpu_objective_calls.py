"""GPU: calls of the objectives that a program makes beside the plain ones: invalid ids and values that are not finite,
rows behind the last, gradients left out or added to, one workspace for changing row counts, empty calls, streams,
captured and replayed calls, more than 2^32 bytes of softmax entries."""
import numpy as np
import pytest
import torch

from objective_util import BF, F4, matrices
from oracle import objectives as oo
from paper_2606_29758_amd import objective, pspo

pytestmark = pytest.mark.gpu
I4, NAN = torch.int32, float("nan")
KINDS = ("policy", "pref", "distill")
OUTPUTS = dict(policy=("loss", "logp_new", "stats", "d_hidden", "d_w_head"),
               pref=("loss", "logp_new", "seq_ratio", "margin", "d_hidden", "d_w_head"),
               distill=("loss", "kl", "d_hidden", "d_w_head"))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


class Inputs:
    """What the three calls take, for up to N rows."""

    def __init__(self, N, d, V, seed=0, R=4, P=3, k=5):
        g = torch.Generator("cuda").manual_seed(seed)
        rand = lambda *s: torch.rand(*s, device="cuda", generator=g)      # noqa: E731
        self.N, self.d, self.V, self.R, self.P, self.k = N, d, V, R, P, k
        self.h, self.w, self.target = matrices(N, d, V, seed)
        self.old = -3 - rand(N)
        self.ref = -3 - rand(N)
        self.weight = 1 + rand(N)
        self.seq = torch.sort((rand(N) * R).int().clamp_max(R - 1)).values.to(I4)
        self.adv = torch.randn(R, device="cuda", generator=g)
        self.cu = torch.sort((rand(R + 1) * N).int()).values.to(I4)
        self.chosen, self.rejected = ((rand(P) * R).int().clamp_max(R - 1).to(I4) for _ in range(2))
        self.ids = (rand(N, k) * V).int().clamp_max(V - 1).to(I4)
        self.t = 3 * torch.randn(N, k, device="cuda", generator=g)

    def call(self, kind, N=None, **kw):
        N = self.N if N is None else N
        if kind == "policy":
            return objective.policy_loss(self.h, self.w, self.target, self.old, self.weight, self.seq, self.adv, N, 0.2, 0.2,
                                         0.01, logp_ref=self.ref, kl_coef=0.1, **kw)
        if kind == "pref":
            cu = self.cu.clamp_max(N)
            return objective.preference_loss(self.h, self.w, self.target, cu, self.chosen, self.rejected, N, 0.1, 0.5,
                                             logp_ref=self.ref, weight=self.weight, **kw)
        return objective.distill_loss(self.h, self.w, self.ids, self.t, N, 0.01, weight=self.weight, **kw)

    def need(self, kind, N, grads=True):
        if kind == "policy":
            return objective.policy_loss_workspace_bytes(N, self.d, self.V, grads)
        if kind == "pref":
            return objective.preference_workspace_bytes(N, self.d, self.V, self.R, self.P, grads)
        return objective.distill_workspace_bytes(N, self.d, self.V, self.k, grads)


def _same(a, b, kind, names=None):
    for n in names or OUTPUTS[kind]:
        x, y = a[n], b[n]
        assert torch.equal(x.nan_to_num(nan=123.0), y.nan_to_num(nan=123.0)) and torch.equal(x.isnan(), y.isnan()), (kind, n)


def _flag():
    return torch.zeros(1, dtype=I4, device="cuda")


SIZES = [(9, 64, 300), (50, 136, 1000), (30, 3592, 200), (200, 64, 1000), (2100, 40, 500)]


@pytest.mark.parametrize("N,d,V", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_the_same_bits_every_time(kind, N, d, V):
    x = Inputs(N, d, V)
    first = x.call(kind)
    assert first["loss"].isfinite() and first["d_hidden"].any() and first["d_w_head"].any()
    for _ in range(2):
        _same(x.call(kind), first, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_one_workspace_for_fewer_rows(kind):
    """A workspace asked for the largest count serves every smaller one, with the bits of one of its own."""
    cap = 600
    for d, V in ((200, 3000), (3592, 300)):
        x = Inputs(cap, d, V)
        ws = torch.empty(x.need(kind, cap), dtype=torch.uint8, device="cuda")
        for N in (1, 15, 16, 17, 32, 33, 48, 49, 64, 65, 100, 129, 257, 300, 511, 600):
            ws.fill_(255)
            a = x.call(kind, N, workspace=ws)
            assert x.need(kind, N) <= ws.numel()
            _same(a, x.call(kind, N), kind)


@pytest.mark.parametrize("N", [10, 40, 100])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_behind_the_last_stay(kind, N):
    x = Inputs(N + 7, 64, 300)
    for dtype in (BF, F4):
        dh, dw = torch.full((N + 7, 64), 7.0, dtype=dtype, device="cuda"), torch.empty(300, 64, dtype=dtype, device="cuda")
        o = x.call(kind, N, d_hidden=dh, d_w_head=dw)
        assert (dh[N:] == 7.0).all() and o["d_hidden"].data_ptr() == dh.data_ptr() and o["d_hidden"].shape == (N, 64)
        assert o["d_w_head"] is dw
        # the rows behind N are not read either
        y = Inputs(N + 7, 64, 300)
        for t in (y.h, y.old, y.ref, y.weight, y.t):
            t[N:] = NAN
        for t in (y.target, y.seq, y.ids):
            t[N:] = 10 ** 6
        _same(y.call(kind, N, d_hidden=torch.empty_like(dh), d_w_head=torch.empty_like(dw)), o, kind)


@pytest.mark.parametrize("N,d,V", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_gradients_left_out(kind, N, d, V):
    """One gradient, or none: the loss and the rows' values within float32 roundings (the sums may be in another order),
    the gradient that is wanted as in the whole call."""
    x = Inputs(N, d, V)
    whole = x.call(kind)
    rows = [n for n in OUTPUTS[kind] if n not in ("d_hidden", "d_w_head")]
    for kw in (dict(want_hidden=False), dict(want_head=False), dict(want_hidden=False, want_head=False)):
        o = x.call(kind, workspace=torch.full((x.need(kind, N, len(kw) == 1),), 255, dtype=torch.uint8, device="cuda"), **kw)
        assert (o["d_hidden"] is None) == ("want_hidden" in kw) and (o["d_w_head"] is None) == ("want_head" in kw)
        for n in rows:
            # sums of up to N terms of log-probs that differ by (d + 2 + 64) 2^-24 of their size (about 20)
            tol = (d + 66) * 2.0 ** -24 * 20 * (N if n in ("seq_ratio", "margin", "stats", "loss") else 1)
            assert ((o[n] - whole[n]).abs() <= tol).all(), n
        for n in ("d_hidden", "d_w_head"):
            if o[n] is not None:
                a, b = o[n].double(), whole[n].double()   # twice the roundings to bf16 of operands and result
                assert (a - b).norm() <= 4 * 2.0 ** -8 * b.norm(), n


@pytest.mark.parametrize("N,d,V", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_head_gradient_added_to(kind, N, d, V):
    x = Inputs(N, d, V)
    alone = x.call(kind, d_w_head=torch.full((V, d), NAN, device="cuda"))["d_w_head"]
    old = torch.randn(V, d, device="cuda") * alone.abs().max()
    both = x.call(kind, d_w_head=old.clone(), accumulate=True)["d_w_head"]
    assert ((both.double() - (old.double() + alone.double())).abs() <= 2.0 ** -24 * (both.abs() + 1e-30)).all()


@pytest.mark.parametrize("N,d,V,hidden,head", [
    (2100, 72, 17003, True, True), (300, 1096, 60001, True, True), (300, 1096, 60001, False, True),
    (130, 2040, 60001, True, True), (1301, 2040, 40001, True, True), (70000, 1024, 2000, True, False)])
def test_tiles_in_chains(N, d, V, hidden, head):
    """Sizes whose work-groups take several tiles in turn, every entry against the formulas in float64.

    With B = 2^-8 for a rounding to bf16: a softmax entry takes one, its row's factor one, the scaled hidden row one; the
    errors of a logit and of the log of the sum, (d + 2) 2^-24 sum |w h| + 2^-18 < 2^-8 each here, move p (and rho, which
    is 1 up to that) by less than three more.  A gradient is off by at most 6 B (1.02 for the second order) of the sum of
    its terms' sizes, and B of itself."""
    h, w, target = matrices(N, d, V, 3)
    g = torch.Generator("cuda").manual_seed(1)
    weight = 1 + torch.rand(N, device="cuda", generator=g)
    weight[::5] = 0
    z = h.double() @ w.double().t()
    lp = z.log_softmax(1)
    del z
    l = lp.gather(1, target.long()[:, None])[:, 0]
    adv = torch.tensor([1.5], device="cuda")
    o = objective.policy_loss(h, w, target, l.float(), weight, torch.zeros(N, dtype=I4, device="cuda"), adv, N, 0.2, 0.2, 1 / 64,
                              want_hidden=hidden, want_head=head)
    assert ((o["logp_new"] - l)[weight > 0].abs() < 2.0 ** -7).all()
    G = lp.exp_()
    G[torch.arange(N, device="cuda"), target.long()] -= 1
    G *= (weight.double() * 1.5 / 64)[:, None]
    size = G.abs()
    B = 2.0 ** -8
    if hidden:
        want, terms = G @ w.double(), size @ w.double().abs()
        assert ((o["d_hidden"].double() - want).abs() <= 6.12 * B * terms + B * want.abs()).all()
    if head:
        want, terms = G.t().contiguous() @ h.double(), size.t().contiguous() @ h.double().abs()
        assert ((o["d_w_head"].double() - want).abs() <= 6.12 * B * terms + B * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("kind", KINDS)
def test_no_rows(kind, dtype):
    x = Inputs(4, 64, 300)
    dw = torch.full((300, 64), 3.0, dtype=dtype, device="cuda")
    o = x.call(kind, 0, d_w_head=dw)
    # (sequences without rows have ratio 0: a pair costs log 2)
    want = 0.5 * x.P * np.log(2) if kind == "pref" else 0.0
    assert abs(float(o["loss"]) - want) < 1e-12 and not dw.any() and o["d_hidden"].shape == (0, 64)
    if dtype == F4:
        dw.fill_(3.0)
        x.call(kind, 0, d_w_head=dw, accumulate=True)
        assert (dw == 3.0).all()


@pytest.mark.parametrize("N,d", [(12, 64), (40, 64), (40, 3592), (150, 64), (2100, 64)])
def test_invalid_ids(N, d):
    """The rows that have them raise the bit and take no part; the others are as if those had weight 0."""
    V = 300
    x, y = Inputs(N, d, V), Inputs(N, d, V)
    bad = torch.tensor([0, 3, N - 1], device="cuda")
    y.weight[bad] = 0.0
    # (a hidden row that is not finite has no effect either)
    x.h[bad], y.h[bad] = NAN, NAN
    x.target[bad] = torch.tensor([-1, V, 2 ** 31 - 1], dtype=I4, device="cuda")
    x.ids[bad, 2] = torch.tensor([V, V + 5, 2 ** 31 - 1], dtype=I4, device="cuda")
    for kind in KINDS:
        err = _flag()
        a, b = x.call(kind, err_flag=err), y.call(kind)
        assert int(err) == 1, kind   # PSPO_DEVERR_TARGET
        value = "kl" if kind == "distill" else "logp_new"
        assert a[value][bad].isnan().all() and (b[value][bad] == 0).all()
        a[value][bad] = 0.0
        _same(a, b, kind)
        assert not a["d_hidden"][bad].any()
    x.target, x.seq[bad] = y.target, torch.tensor([-1, x.R, 2 ** 30], dtype=I4, device="cuda")
    err = _flag()
    a = x.call("policy", err_flag=err)
    assert int(err) == 8   # PSPO_DEVERR_SEQ_ID
    a["logp_new"][bad] = 0.0
    _same(a, y.call("policy"), "policy")


def test_invalid_pairs_and_offsets():
    N, V = 100, 300
    x = Inputs(N, 64, V, R=5, P=4)
    x.cu = torch.tensor([0, 20, 40, 60, 80, 95], dtype=I4, device="cuda")
    x.chosen = torch.tensor([0, 5, 2, -1], dtype=I4, device="cuda")
    x.rejected = torch.tensor([1, 1, 2 ** 30, 3], dtype=I4, device="cuda")
    err = _flag()
    a = x.call("pref", err_flag=err)
    assert int(err) == 8 and a["margin"][1:].isnan().all() and a["margin"][0].isfinite()
    x.chosen, x.rejected, x.P = x.chosen[:1].clone(), x.rejected[:1].clone(), 1
    _same(a, x.call("pref"), "pref", ("loss", "logp_new", "seq_ratio", "d_hidden", "d_w_head"))
    assert not a["d_hidden"][40:].any() and a["d_hidden"][:40].any()
    # offsets that decrease, or lie outside the rows: the bit, and nothing out of range
    for cu in ([0, 50, 30, 60, 80, 95], [-5, 20, 40, 60, 80, 95], [0, 20, 40, 60, 80, 101], [2 ** 31 - 1, -2 ** 31, 7, 7, 7, 7]):
        for big in (False, True):   # in one work-group, and by the kernels of many pairs
            err = _flag()
            p = torch.zeros(2 ** 18 if big else 1, dtype=I4, device="cuda")
            o = objective.preference_loss(x.h, x.w, x.target, torch.tensor(cu, dtype=I4, device="cuda"), p, p + 1, N, 0.1,
                                          0.5, err_flag=err)
            torch.cuda.synchronize()
            assert int(err) & 8 and o["loss"].isfinite(), cu


def test_many_pairs_as_few():
    """The kernels of many pairs and the one of few give the same loss and gradients, to float64 roundings."""
    x = Inputs(300, 64, 500, R=8, P=6)
    few = x.call("pref")
    times = 2 ** 15
    x.chosen, x.rejected = x.chosen.repeat(times), x.rejected.repeat(times)
    many = objective.preference_loss(x.h, x.w, x.target, x.cu, x.chosen, x.rejected, 300, 0.1, 0.5 / times, logp_ref=x.ref,
                                     weight=x.weight)
    assert abs(float(many["loss"] - few["loss"])) < 1e-10 * float(few["loss"])
    assert torch.equal(many["margin"][:6], few["margin"])
    for n in ("d_hidden", "d_w_head"):   # factors that differ in their last float64 bits may round to the other side
        assert ((many[n].float() - few[n].float()).abs() <= 2.0 ** -6 * few[n].float().abs() + 1e-30).all()


@pytest.mark.parametrize("N", [12, 40, 150, 2100])
def test_values_that_are_not_finite(N):
    for kind in KINDS:
        for spoil in ("h", "weight", "ref", "old", "t", "adv"):
            if spoil in (("ref", "old", "adv") if kind == "distill" else ("t", "old", "adv") if kind == "pref" else ("t",)):
                continue
            x = Inputs(N, 64, 300)
            getattr(x, spoil).view(-1)[1] = NAN
            if kind == "pref":   # (row 1 has to stand in a sequence that a pair names)
                x.cu = torch.tensor([0, N // 2, N, N, N], dtype=I4, device="cuda")
                x.chosen, x.rejected = (torch.tensor([v] * x.P, dtype=I4, device="cuda") for v in (0, 1))
            if kind == "policy" and spoil == "adv":
                x.adv.fill_(NAN)
            err = _flag()
            o = x.call(kind, err_flag=err)
            assert int(err) == 16 and not o["loss"].isfinite(), (kind, spoil)


@pytest.mark.parametrize("N", [12, 40, 150, 2100])
def test_gradients_past_float32(N):
    """Logits of 0, so that the log-probs and losses are small; at a temperature of 1e-36 the factors of p (weight 1 to 2
    times 0.01, or beta 0.1 and scale 0.5, times 1e36) pass 3.5e38 from weights of 1e6 on."""
    for kind in KINDS:
        x = Inputs(N, 64, 300)
        x.h.zero_()
        x.old.fill_(-np.log(300))
        x.adv.fill_(1)
        x.cu = torch.tensor([0, N // 2, N, N, N], dtype=I4, device="cuda")
        x.chosen, x.rejected = (torch.tensor([v] * x.P, dtype=I4, device="cuda") for v in (0, 1))
        for many, want in ((1.0, 0), (1e6, 16)):
            err = _flag()
            x.weight.mul_(many)
            if kind == "pref":   # equal weights: the log ratios of N // 2 and of N - N // 2 rows differ by one row's at most
                x.weight.fill_(many)
                x.ref.fill_(-np.log(300))
            if kind == "distill":
                x.t.fill_(0)
            call = dict(temperature=1e-36, err_flag=err)
            o = x.call(kind, **call)
            assert int(err) == want and bool(o["loss"].isfinite()), (kind, many)


@pytest.mark.parametrize("kind", KINDS)
def test_streams(kind):
    """Calls on several streams at once, each with a workspace of its own, give the bits of calls one after another."""
    xs = [Inputs(N, 136, 2000, seed=s) for s, N in enumerate((14, 60, 300, 2100))]
    want = [x.call(kind) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [None] * len(xs)
    for rep in range(3):
        for i, (x, s) in enumerate(zip(xs, streams)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = x.call(kind)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            _same(a, b, kind)


@pytest.mark.parametrize("N,d", [(14, 64), (60, 136), (60, 3592), (300, 64), (2100, 40)])
@pytest.mark.parametrize("kind", KINDS)
def test_graphs(kind, N, d):
    """Captured once, replayed with eager work and changed inputs between: every replay gives the eager call's bits."""
    x, other = Inputs(N, d, 700), Inputs(N, d, 700, seed=5)
    ws = torch.empty(x.need(kind, N), dtype=torch.uint8, device="cuda")
    dh, dw = torch.empty(N, d, dtype=BF, device="cuda"), torch.empty(700, d, device="cuda")
    kw = dict(workspace=ws, d_hidden=dh, d_w_head=dw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x.call(kind, **kw)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = x.call(kind, **kw)
    for rep in range(4):
        x.h.copy_(other.h if rep % 2 else Inputs(N, d, 700, seed=9).h)
        want = {n: t.clone() for n, t in x.call(kind).items() if isinstance(t, torch.Tensor)}
        want["d_w_head"] = x.call(kind, d_w_head=torch.empty_like(dw))["d_w_head"].clone()
        other.call(kind)
        ws.fill_(255)
        for n in OUTPUTS[kind]:
            out[n].fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _same(out, want, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_debug_mode(kind, monkeypatch):
    for N in (14, 100):
        x = Inputs(N, 64, 300)
        want = x.call(kind)
        monkeypatch.setenv("PSPO_DEBUG", "1")
        _same(x.call(kind), want, kind)
        monkeypatch.delenv("PSPO_DEBUG")


def test_refused_calls_leave_everything():
    x = Inputs(20, 64, 300)
    dw = torch.full((300, 64), 3.0, device="cuda")
    for kind in KINDS:
        for kw in (dict(temperature=0.0), dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
            with pytest.raises(pspo.PspoError):
                x.call(kind, d_w_head=dw, **kw)
    torch.cuda.synchronize()
    assert (dw == 3.0).all()


def test_more_than_2_to_32_bytes_of_entries():
    """15,001 rows of 151936 entries (4.6 GB): the last rows' values and gradients, and the head's, against float32 torch."""
    N, d, V = 15001, 64, 151936
    x = Inputs(N, d, V)
    err = _flag()
    o = x.call("distill", err_flag=err)
    assert int(err) == 0
    hf, wf = x.h.float(), x.w.float()
    dw = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    dh, kl = torch.empty(N, d, device="cuda"), torch.empty(N, device="cuda")
    for a in range(0, N, 1000):
        s = slice(a, min(a + 1000, N))
        lp = torch.log_softmax(hf[s] @ wf.T, 1)
        q = torch.softmax(x.t[s], 1)
        G = lp.exp().scatter_add_(1, x.ids[s].long(), -q)
        kl[s] = (q * (q.log() - lp.gather(1, x.ids[s].long()))).sum(1)   # (repeated ids: next to never at this V)
        G = G * (0.01 * x.weight[s])[:, None]
        dh[s] = G @ wf
        dw += (G.T @ hf[s]).double()
    # roundings to bf16: the entries, the scaled rows, the results, 2^-8 each at most; sums are longer than one entry
    for got, want in ((o["d_hidden"], dh), (o["d_w_head"], dw), (o["d_hidden"][-100:], dh[-100:])):
        assert (got.double() - want.double()).norm() <= 3 * 2.0 ** -8 * want.double().norm()
    there = (x.ids.sort(1).values.diff(dim=1) != 0).all(1)
    assert (o["kl"] - kl)[there].abs().max() <= 2 * (d + 66) * 2.0 ** -24 * 20
