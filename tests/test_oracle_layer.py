"""The float64 oracle of the layer operators against independent statements: central differences,
known answers of the generator, the rotation's invariants, torch's float64 autograd."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as ol


def _diff(f, x, dout, h=1e-6):
    """Central differences of sum(f(x) * dout) by every entry of x."""
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = ((f(a) - f(b)) * dout).sum() / (2 * h)
    return g


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_head_norm_gradient_is_the_difference(interleaved, norm):
    rng = np.random.default_rng(1)
    x, dout = rng.normal(size=(3, 2, 24)), rng.normal(size=(3, 2, 24))
    w = rng.normal(size=24) if norm else None
    pos, inv = np.array([0, 7, 131071]), np.array([1.0, 0.5, 0.1, 0.03, 0.01, 0.003, 0.001, 0.0001])
    dx, dw = ol.qk_norm_rope_bwd(dout, x, w, pos, inv, 1e-6, interleaved, norm)
    f = lambda a: ol.qk_norm_rope(a, w, pos, inv, 1e-6, interleaved, norm)   # noqa: E731
    assert np.allclose(dx, _diff(f, x, dout), rtol=1e-6, atol=1e-7)
    if norm:
        fw = lambda a: ol.qk_norm_rope(x, a, pos, inv, 1e-6, interleaved, norm)   # noqa: E731
        assert np.allclose(dw, _diff(fw, w, dout), rtol=1e-6, atol=1e-7)


def test_rotation_depends_on_distance_and_keeps_lengths():
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(1, 1, 32)), rng.normal(size=(1, 1, 32))
    inv = 10000.0 ** (-np.arange(16) / 16)
    for il in (False, True):
        at = lambda x, p: ol.rotate(x, [p], inv, il)   # noqa: E731
        assert np.isclose((at(q, 9) * at(k, 4)).sum(), (at(q, 105) * at(k, 100)).sum())
        assert np.isclose(np.linalg.norm(at(q, 77)), np.linalg.norm(q))
        assert np.array_equal(at(q, 0), q)
        assert np.allclose(ol.rotate(at(q, 5), [5], inv, il, back=True), q)


def test_positions():
    pos = ol.positions([0, 0, 2, 2, 2, 5, -1], [0, 2, 2, 5], [10, 20, 30], 7)
    assert pos.tolist() == [10, 11, 30, 31, 32, 0, 0]


def test_mask_from_the_generators_known_answer():
    """Row 0 of counter (0, 1, 0, 0) under key 0: the sixteen-bit words in order, low half first."""
    words = ol.philox4x32((0, 1, 0, 0), (0, 0))
    halves = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    m = ol.dropout_mask([0], 8, 0.5, 0, 0)[0]
    assert m.tolist() == [h < 32768 for h in halves]


def test_mask_rate_and_dropped_values():
    m = ol.dropout_mask(range(64), 256, 0.25, 12345, 7)
    # 16384 draws at 3/4: standard deviation 0.0034
    assert abs(m.mean() - 0.75) < 4 * 0.0034
    assert ol.dropout_mask([3], 64, 0.0, 1, 0).all()
    assert ol.keep_threshold(0.999999) == 1 and ol.keep_threshold(0.0) == 65536
    y = ol.dropout_add(np.array([[np.nan, 2.0]]), None, np.array([[False, True]]), 0.5)
    assert y.tolist() == [[0.0, 4.0]]


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_gated_ffn_against_autograd(act):
    rng = np.random.default_rng(3)
    x, wg, wu, wd = (rng.normal(size=s) for s in ((5, 8), (16, 8), (16, 8), (8, 16)))
    dy = rng.normal(size=(5, 8))
    t = [torch.from_numpy(a).requires_grad_() for a in (x, wg, wu, wd)]
    F = torch.nn.functional
    g = F.linear(t[0], t[1])
    a = F.silu(g) if act == "silu" else F.gelu(g, approximate="tanh")
    y = F.linear(a * F.linear(t[0], t[2]), t[3])
    ref = torch.autograd.grad(y, t, torch.from_numpy(dy))
    got_y, pre = ol.gated_ffn(x, wg, wu, wd, act)
    assert np.allclose(got_y, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    assert np.allclose(pre[:, :16], x @ wg.T) and np.allclose(pre[:, 16:], x @ wu.T)
    for a, b in zip(ol.gated_ffn_bwd(dy, x, wg, wu, wd, act), ref):
        assert np.allclose(a, b.numpy(), rtol=1e-10, atol=1e-12)


def test_gated_ffn_gradient_is_the_difference():
    rng = np.random.default_rng(4)
    x, wg, wu, wd = (rng.normal(size=s) for s in ((2, 8), (8, 8), (8, 8), (8, 8)))
    dy = rng.normal(size=(2, 8))
    dx, dwg, _, _ = ol.gated_ffn_bwd(dy, x, wg, wu, wd, "gelu_tanh")
    assert np.allclose(dx, _diff(lambda a: ol.gated_ffn(a, wg, wu, wd, "gelu_tanh")[0], x, dy), rtol=1e-5, atol=1e-7)
    assert np.allclose(dwg, _diff(lambda a: ol.gated_ffn(x, a, wu, wd, "gelu_tanh")[0], wg, dy), rtol=1e-5, atol=1e-7)


def test_activation_far_out():
    for act in ("silu", "gelu_tanh"):
        a, da = ol.activation(np.array([-500.0, 500.0]), act)
        assert np.allclose(a, [0.0, 500.0], atol=1e-100) and np.allclose(da, [0.0, 1.0], atol=1e-100)
