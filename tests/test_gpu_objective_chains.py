"""GPU: work-groups that take several tiles in turn, with float32 gradients, alone and added to, and with lists of ids:
the stores, and the loads of what is added to, that run while the next tile's first stages are on their way.

Every entry against the formulas in float64.  With B = 2^-8 for a rounding to bf16: a softmax entry takes one, its row's
factor one, the scaled hidden row one; the errors of a logit and of the log of the sum, (d + 2) 2^-24 sum |w h| + 2^-18
< 2^-8 each here, move p (and rho, which is 1 up to that) by less than three more; a float32 sum of n terms takes n 2^-24.
A gradient is off by at most 6 B + n 2^-24 (1.02 for the second order) of the sum of its terms' sizes, where an entry at
an id of a list counts p + q.
"""
import pytest
import torch

from objective_util import BF, F4, matrices
from paper_2606_29758_amd import objective

pytestmark = pytest.mark.gpu
I4, NAN, B, U = torch.int32, float("nan"), 2.0 ** -8, 2.0 ** -24

# N, d, V: the forward product and the head's gradient in chains, in one launch with d_hidden; the head's alone; d_hidden's
# alone; a micro-batch of a real head; an odd vocabulary with lists
SIZES = [(2100, 72, 17003, True, True), (300, 1096, 60001, True, True), (300, 1096, 60001, False, True),
         (130, 2040, 60001, True, True), (70000, 1024, 2000, True, False), (777, 1536, 151936, True, True),
         (1301, 520, 32003, True, True), (1301, 520, 32003, False, True)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


def _case(kind, N, d, V):
    """The call, and G with the sizes of its terms (float64)."""
    h, w, target = matrices(N, d, V, 4)
    g = torch.Generator("cuda").manual_seed(2)
    weight = 1 + torch.rand(N, device="cuda", generator=g)
    weight[::5] = 0
    lp = (h.double() @ w.double().t()).log_softmax(1)
    row = torch.arange(N, device="cuda")
    if kind == "policy":
        l = lp[row, target.long()]
        adv, seq = torch.tensor([1.5], device="cuda"), torch.zeros(N, dtype=I4, device="cuda")
        call = lambda **kw: objective.policy_loss(h, w, target, l.float(), weight, seq, adv, N, 0.2, 0.2, 1 / 64, **kw)   # noqa: E731
        G = lp.exp_()
        G[row, target.long()] -= 1
        G *= (weight.double() * 1.5 / 64)[:, None]
        return call, h, w, G, G.abs()
    k = 50
    ids = (target[:, None].long() + torch.arange(k, device="cuda") * torch.randint(1, V // k, (N, 1), device="cuda", generator=g)) % V
    ids[:, 7] = -1
    t = 2 * torch.randn(N, k, device="cuda", generator=g)
    q = t.double()
    q[:, 7] = -float("inf")
    q = q.softmax(1)
    i4 = ids.to(I4)
    call = lambda **kw: objective.distill_loss(h, w, i4, t, N, 1 / 64, weight=weight, **kw)   # noqa: E731
    G = lp.exp_()
    size = G.scatter_add(1, ids.clamp_min(0), q)
    G.scatter_add_(1, ids.clamp_min(0), -q)
    c = (weight.double() / 64)[:, None]
    return call, h, w, G.mul_(c), size.mul_(c)


@pytest.mark.parametrize("kind", ["policy", "distill"])
@pytest.mark.parametrize("N,d,V,hidden,head", SIZES)
def test_float32_gradients(kind, N, d, V, hidden, head):
    call, h, w, G, size = _case(kind, N, d, V)
    new = lambda n, fill: torch.full((n, d), fill, dtype=F4, device="cuda")   # noqa: E731
    want_of = dict(want_hidden=hidden, want_head=head)
    kw = lambda fill: dict(want_of, **({"d_hidden": new(N, fill)} if hidden else {}), **({"d_w_head": new(V, fill)} if head else {}))   # noqa: E731
    o = call(**kw(NAN))
    if hidden:
        want, terms = G @ w.double(), size @ w.double().abs()
        assert ((o["d_hidden"].double() - want).abs() <= 1.02 * (6 * B + V * U) * terms).all()
    if head:
        want, terms = G.t().contiguous() @ h.double(), size.t().contiguous() @ h.double().abs()
        assert ((o["d_w_head"].double() - want).abs() <= 1.02 * (6 * B + N * U) * terms).all()
        del want, terms
        # the same bits again, and added to what stands there: one rounding to float32 beside the sum
        for _ in range(2):
            again = call(**kw(1.0))
            assert torch.equal(again["d_w_head"], o["d_w_head"]) and torch.equal(again["loss"], o["loss"])
        old = torch.randn(V, d, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) * o["d_w_head"].abs().max()
        got = call(**dict(kw(NAN), d_w_head=old.clone()), accumulate=True)["d_w_head"].double()
        both = old.double() + o["d_w_head"].double()
        assert ((got - both).abs() <= U * (both.abs() + 1e-30)).all()
    # bf16 gradients are the float32 ones rounded
    b = call(**want_of)
    for n in ("d_hidden", "d_w_head"):
        if o[n] is not None:
            assert b[n].dtype == BF and torch.equal(b[n], o[n].to(BF)), n
