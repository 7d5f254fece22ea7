"""GPU: the gated feed-forward block at sizes whose plans take the tiles, rings and K parts that small calls do
not (layer_sizes.py; test_layer_paths_cpu.py holds the list against the plans), on rows and columns of every tile.

The reference is float64 on the formulas: every entry of the sampled tokens' y, pre-activations and dx, and every
entry of the sampled rows of dw_gate, dw_up and columns of dw_down.  One token and one feed-forward entry are
drawn in each block of 64, beside the first and the last.  The bounds are those of test_gpu_layer_ffn.py,
carried through the formulas entry by entry (u = 2^-24, b = 2^-8).  At these lengths they are a large part of an
entry, so spans of 64 entries of a row are held in 2-norm besides: a rounding to bf16 is off by 2^-8 / sqrt(3)
rms at most, those of a sum's terms are independent of each other and of the terms' signs (random weights), and
at most two stand between the inputs and a result, sqrt(2/3) 2^-8 = 3.2e-3; 2^-6 is allowed, and one stage of 64
left out of the longest sum here (28,672 terms) would be 4.7e-2.
"""
import pytest
import torch

from layer_sizes import FFN_PATHS
from paper_2606_29758_amd import layer

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
BF, F4 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _inputs(N, d, f, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    new = lambda *s, k=1.0: (torch.randn(*s, device="cuda", generator=g) * k).to(BF)   # noqa: E731
    return (new(N, d), new(f, d, k=1.5 / d ** 0.5), new(f, d, k=1 / d ** 0.5), new(d, f, k=1 / f ** 0.5),
            new(N, d, k=0.1)), g


def _sample(n, g):
    at = torch.arange(0, n, 64, device="cuda")
    at = at + torch.randint(0, 64, at.shape, device="cuda", generator=g)
    return torch.unique(torch.cat([at.clamp(max=n - 1), torch.tensor([0, n - 1], device="cuda")]))


def _act(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    a = (2 / torch.pi) ** 0.5
    t = torch.tanh(a * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 0.134145 * g * g)


def _sum(n):
    return (n + 2) * U


class Inner:
    """g, u, h, dg, du of tokens x, dy (rows) by feed-forward entries (rows of wg, wu, columns of wd), with bounds."""

    def __init__(self, x, dy, wg, wu, wd, act):
        d = x.shape[1]
        self.g, self.u = x @ wg.T, x @ wu.T
        self.eg, self.eu = _sum(d) * (x.abs() @ wg.abs().T), _sum(d) * (x.abs() @ wu.abs().T)
        g, u, eg, eu = self.g, self.u, self.eg, self.eu
        a, da = _act(g, act)
        ea = 1.13 * eg + 32 * U * g.abs()
        eda = 0.8 * eg + 32 * U * (1 + a.abs() + g.abs())
        self.h = a * u
        self.eh = (ea * u.abs() + a.abs() * eu + ea * eu) * (1 + B) + B * self.h.abs()
        dh = dy @ wd
        edh = _sum(d) * (dy.abs() @ wd.abs())
        self.dg, self.du = dh * u * da, dh * a
        self.edg = (edh * (u * da).abs() + dh.abs() * (eu * da.abs() + u.abs() * eda) + 4 * U * self.dg.abs()) * (
            1 + 1e-3) * (1 + B) + B * self.dg.abs()
        self.edu = (edh * a.abs() + dh.abs() * ea + 4 * U * self.du.abs()) * (1 + 1e-3) * (1 + B) + B * self.du.abs()


def _product(p, ep, q, n):
    return p @ q, ep @ q.abs() + _sum(n) * ((p.abs() + ep) @ q.abs())


def _close(got, want, err, bf16, what):
    e = (got.double() - want).abs()
    tol = (err * (1 + B) + B * want.abs() if bf16 else err) + 1e-30
    assert (e <= tol).all(), (what, float((e / tol).max()))
    pad = torch.nn.functional.pad
    span = lambda t: pad(t, (0, -t.shape[1] % 64)).unflatten(1, (-1, 64)).norm(dim=2)   # noqa: E731
    off, size = span(e), span(want)
    assert (off <= 2.0 ** -6 * size).all(), (what, float((off / size).max()))


@pytest.mark.parametrize("N,d,f,act", [(*s, ("silu", "gelu_tanh")[i % 2]) for i, s in enumerate(FFN_PATHS)])
def test_paths(N, d, f, act):
    (x, wg, wu, wd, dy), gen = _inputs(N, d, f, 17 * N + d + f)
    kept = layer.gated_ffn(x, wg, wu, wd, N, act=act, keep=True)
    plain = layer.gated_ffn(x, wg, wu, wd, N, act=act)
    assert torch.equal(plain["y"], kept["y"])
    names = ("dx", "dw_gate", "dw_up", "dw_down")
    o = layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, act=act, preact=kept["preact"])
    again = layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, act=act)
    assert all(torch.equal(o[k], again[k]) for k in names)   # the pre-activations computed again are the same
    dw = tuple(torch.full(s, 7.0, device="cuda") for s in ((f, d), (f, d), (d, f)))
    o32 = layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, act=act, preact=kept["preact"], dw=dw)
    once = [t.clone() for t in dw]
    layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, act=act, preact=kept["preact"], dw=dw, accumulate=True)
    assert all(torch.equal(t, 2 * v) for t, v in zip(dw, once))   # the same sum added to itself: exact
    assert torch.equal(o32["dx"], o["dx"])
    assert all(torch.equal(v.to(BF), o[k]) for k, v in zip(names[1:], once))   # one rounding of the same sums

    w = [t.double() for t in (wg, wu, wd)]
    rows, cols = _sample(N, gen), _sample(f, gen)
    r = Inner(x[rows].double(), dy[rows].double(), *w, act)
    _close(kept["preact"][rows], torch.cat([r.g, r.u], 1), torch.cat([r.eg, r.eu], 1), False, "preact")
    _close(kept["y"][rows], *_product(r.h, r.eh, w[2].T, f), True, "y")
    v1, e1 = _product(r.dg, r.edg, w[0], 2 * f)
    v2, e2 = _product(r.du, r.edu, w[1], 2 * f)
    _close(o["dx"][rows], v1 + v2, e1 + e2, True, "dx")
    del r, v1, v2, e1, e2
    x64, dy64 = x.double(), dy.double()
    c = Inner(x64, dy64, w[0][cols], w[1][cols], w[2][:, cols].contiguous(), act)
    for name, got, (v, e) in (("dw_gate", once[0][cols], _product(c.dg.T, c.edg.T, x64, N + 66)),
                              ("dw_up", once[1][cols], _product(c.du.T, c.edu.T, x64, N + 66)),
                              ("dw_down", once[2][:, cols].T, _product(c.h.T, c.eh.T, dy64, N + 66))):
        _close(got, v, e, False, name)
