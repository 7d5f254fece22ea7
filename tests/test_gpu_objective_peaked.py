"""GPU: rows whose softmax is all but one entry.  With o a row's first id and rest = sum over the others of exp(z_v - z_o),
log p_o = -log1p(rest) and 1 - p_o = rest / (1 + rest), which lose no digits however small rest is; the calls have to
keep them: a log-prob is never positive, and the entry of G at o has the size of the row's others together.

Each row has a column of the hidden state to itself (1 there, the head 0), in which d_w_head holds its G.

Bounds, u = 2^-24 and B = 2^-8: a term of rest is off by e = (d + 2) u s |h| |w_v| (its float32 logit), 8 u s |h| |w_o|
(groups of eight products in float32) and 8 u (|z_o - z_v| + 1) (its exponential), their sums by 80 u more; an entry of G by
2 B for its rounding and that of the row's factor, B for the factor in d_w_head, and the error of p.  Second order: 1.02.
"""
import math

import pytest
import torch

from objective_util import BF, F4
from paper_2606_29758_amd import objective

pytestmark = pytest.mark.gpu
I4, U, B = torch.int32, 2.0 ** -24, 2.0 ** -8
OWN = 64   # columns that the head reads


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


class Peaked:
    def __init__(self, N, d, V, T, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.N, self.d, self.V, self.T = N, d, V, T
        w = torch.zeros(V, d, device="cuda")
        w[:, :OWN] = torch.randn(V, OWN, device="cuda", generator=g) * 0.15
        self.w = w.to(BF)
        self.o = torch.randint(0, V, (N,), device="cuda", generator=g)
        up = self.w[self.o].float()
        top = T * (math.log(V) + 15 + 15 * torch.rand(N, 1, device="cuda", generator=g))
        h = torch.zeros(N, d, device="cuda")
        h[:, :OWN] = torch.randn(N, OWN, device="cuda", generator=g)
        h += up * top / up.square().sum(1, keepdim=True)
        row = torch.arange(N, device="cuda")
        h[row, OWN + row] = 1
        self.h, self.row = h.to(BF), row
        hd, wd = self.h.double(), self.w.double()
        self.z = hd @ wd.t().contiguous() / T
        self.size = hd.abs() @ wd.abs().t().contiguous() / T
        zo = self.z[row, self.o]
        self.x = torch.exp(self.z - zo[:, None])          # exp(z_v - z_o)
        others = self.x.clone()
        others[row, self.o] = 0
        rest = others.sum(1)
        assert rest.median() < 1e-3 and rest.min() < 1e-6
        self.l, self.left = -torch.log1p(rest), rest / (1 + rest)
        self.p = self.x / (1 + rest)[:, None]
        e_own = 8 * U * self.size[row, self.o]
        self.e = 1.02 * ((d + 2) * U * self.size + e_own[:, None] + 8 * U * ((zo[:, None] - self.z).abs() + 1) + 80 * U)
        self.e_rest = (others * self.e).sum(1) / rest    # relative, of rest
        self.e_l = self.left * self.e_rest + U * self.l.abs()

    def G(self, o):
        """The rows' logit gradient as d_w_head holds it: [N, V]."""
        assert o["d_w_head"].dtype == F4
        return o["d_w_head"][:, OWN:OWN + self.N].t().double()

    def check_target(self, o, delta, e_delta):
        """The log-probs, and G where d loss / d l = delta."""
        l = o["logp_new"].double()
        assert (l <= 0).all(), l.max()
        assert ((l - self.l).abs() <= 1.02 * self.e_l).all(), ((l - self.l).abs() / self.e_l).max()
        if o["d_w_head"] is None:
            return
        s, row = 1 / self.T, self.row
        want = -s * delta[:, None] * self.p
        tol = s * delta.abs()[:, None] * self.p * (3 * B + self.e + 8 * U) + s * e_delta[:, None] * self.p
        want[row, self.o] = s * delta * self.left
        tol[row, self.o] = s * (delta.abs() * self.left * (2 * B + self.e_rest + 8 * U) + e_delta * self.left)
        off = (self.G(o) - want).abs() / (1.03 * tol + 1e-37)
        assert (off <= 1).all(), (off.max(), off[row, self.o].max())


CASES = [(3, 72, 300), (16, 80, 1000), (40, 104, 5000), (5, 3592, 400), (150, 216, 1000), (70, 2048, 700), (300, 1096, 60001),
         (2100, 2168, 700)]   # both kernels of few rows, float32 logits, tiles, K parts, chains of tiles, rows by waves


@pytest.mark.parametrize("T", [1.0, 0.5])
@pytest.mark.parametrize("N,d,V", CASES)
def test_policy(N, d, V, T):
    x = Peaked(N, d, V, T, seed=N)
    old = x.l.float()
    one = torch.ones(N, device="cuda")
    call = lambda **kw: objective.policy_loss(x.h, x.w, x.o.to(I4), old, one, torch.zeros(N, dtype=I4, device="cuda"),   # noqa: E731
                                              one[:1].contiguous(), N, 0.2, 0.2, 1.0, temperature=T, **kw)
    delta = -torch.exp(x.l - old.double())
    x.check_target(call(d_w_head=torch.empty(V, d, device="cuda")), delta, delta.abs() * (1.02 * x.e_l + 4 * U))
    x.check_target(call(want_hidden=False, want_head=False), delta, None)


@pytest.mark.parametrize("T", [1.0, 0.5])
@pytest.mark.parametrize("N,d,V", CASES)
def test_preference(N, d, V, T):
    x = Peaked(N, d, V, T, seed=N + 1)
    half, beta = N // 2, 0.1
    ints = lambda *v: torch.tensor(v, dtype=I4, device="cuda")   # noqa: E731
    call = lambda **kw: objective.preference_loss(x.h, x.w, x.o.to(I4), ints(0, half, N), ints(0), ints(1), N, beta, 1.0,   # noqa: E731
                                                  temperature=T, **kw)
    u = x.l[:half].sum() - x.l[half:].sum()
    coef = -beta * torch.sigmoid(-beta * u)
    delta = torch.where(x.row < half, coef, -coef)
    e_delta = beta * beta / 4 * x.e_l.sum() + 4 * U * delta.abs()
    o = call(d_w_head=torch.empty(V, d, device="cuda"))
    x.check_target(o, delta, e_delta)
    assert (o["seq_ratio"] <= 0).all()
    for r, rows in enumerate((slice(0, half), slice(half, N))):
        assert (o["seq_ratio"][r].double() - x.l[rows].sum()).abs() <= 1.02 * x.e_l[rows].sum() + U * x.l[rows].sum().abs()
    x.check_target(call(want_hidden=False, want_head=False), delta, None)


@pytest.mark.parametrize("T", [1.0, 0.5])
@pytest.mark.parametrize("N,d,V", CASES)
def test_distillation(N, d, V, T):
    """Lists whose first id (there twice) has all but e^-9 to e^-20 of the teacher's probability too: p - q there is
    (1 - q) - (1 - p).  A divergence is the sum of q (log q - log p), terms of both signs: its bound goes by their errors."""
    x = Peaked(N, d, V, T, seed=N + 2)
    s, row = 1 / T, x.row
    ids = torch.stack([x.o, (x.o + 1) % V, (x.o + 2) % V, x.o, torch.full_like(x.o, -1)], 1)
    low = -9 - 11 * torch.rand(N, 2, device="cuda", generator=torch.Generator("cuda").manual_seed(N))
    t = torch.stack([torch.zeros_like(low[:, 0]), low[:, 0], low[:, 1], torch.zeros_like(low[:, 0]) - 1,
                     torch.zeros_like(low[:, 0])], 1)
    y = torch.exp(t[:, :4].double() / T)
    q = torch.stack([y[:, 0] + y[:, 3], y[:, 1], y[:, 2]], 1) / y.sum(1, keepdim=True)
    away = (y[:, 1] + y[:, 2]) / y.sum(1)
    p, z = x.p.gather(1, ids[:, :3]), x.z.gather(1, ids[:, :3])
    lp = z - z[:, :1] + x.l[:, None]
    lq = torch.log(q)
    lq[:, 0] = torch.log1p(-away)
    e_lp = 8 * U * (x.size.gather(1, ids[:, :3]) + x.size[row, x.o][:, None]) + (x.left * x.e_rest)[:, None]
    e_lp[:, 0] = x.left * x.e_rest
    e_kl = (q * (1.02 * e_lp + 4e-16 * (1 + z.abs()))).sum(1)
    want_kl = (q * (lq - lp)).sum(1)
    alone = objective.distill_loss(x.h, x.w, ids.to(I4), t, N, 1.0, temperature=T, want_hidden=False, want_head=False)
    o = objective.distill_loss(x.h, x.w, ids.to(I4), t, N, 1.0, temperature=T, d_w_head=torch.empty(V, d, device="cuda"))
    for got in (alone, o):
        assert ((got["kl"].double() - want_kl).abs() <= e_kl + U * want_kl.abs()).all()
        assert abs(float(got["loss"]) - float(want_kl.sum())) <= float(e_kl.sum())
    want = s * x.p
    tol = s * x.p * (3 * B + x.e + 8 * U)
    for j in (1, 2):
        want[row, ids[:, j]] = s * (p[:, j] - q[:, j])
        tol[row, ids[:, j]] = s * ((p[:, j] - q[:, j]).abs() * 2 * B + p[:, j] * x.e[row, ids[:, j]] + 8 * U * (p[:, j] + q[:, j]))
    want[row, x.o] = s * (away - x.left)
    tol[row, x.o] = s * ((away - x.left).abs() * 2 * B + x.left * (x.e_rest + 8 * U) + 8 * U * away)
    off = (x.G(o) - want).abs() / (1.03 * tol + 1e-37)
    assert (off <= 1).all(), (off.max(), off[row, x.o].max())
