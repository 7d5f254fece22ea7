"""GPU: calls of the layer operators that a program makes beside the plain ones: one workspace for changing
token counts, empty calls, refused arguments."""
import pytest
import torch

from paper_2606_29758_amd import layer

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _ffn(N, d, f, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    new = lambda *s, k=1.0: (torch.randn(*s, device="cuda", generator=g) * k).to(BF)   # noqa: E731
    return (new(N, d), new(f, d, k=1 / d ** 0.5), new(f, d, k=1 / d ** 0.5), new(d, f, k=1 / f ** 0.5),
            new(N, d, k=0.1))


def test_one_workspace_for_fewer_tokens():
    """A workspace asked for the largest count serves every smaller one, with the same bits as one of its own."""
    cap, d, f = 1025, 1000, 4104
    x, wg, wu, wd, dy = _ffn(cap, d, f)
    fwd = torch.empty(layer.gated_ffn_workspace_bytes(cap, d, f), dtype=torch.uint8, device="cuda")
    bwd = torch.empty(layer.gated_ffn_workspace_bytes(cap, d, f, True, True), dtype=torch.uint8, device="cuda")
    for N in (1, 20, 64, 65, 128, 129, 200, 257, 400, 513, 777, 1000, 1024, 1025):
        a = layer.gated_ffn(x, wg, wu, wd, N, keep=True, workspace=fwd)
        b = layer.gated_ffn(x, wg, wu, wd, N, keep=True)
        assert torch.equal(a["y"], b["y"]) and torch.equal(a["preact"], b["preact"]), N
        p = layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, preact=a["preact"], workspace=bwd)
        q = layer.gated_ffn_bwd(dy, x, wg, wu, wd, N, preact=a["preact"])
        assert all(torch.equal(p[k], q[k]) for k in ("dx", "dw_gate", "dw_up", "dw_down")), N


def test_an_empty_backward_without_a_workspace():
    """No tokens ask for 0 bytes: the C call takes NULL and writes (or adds) zeros."""
    lib, d, f = layer.load(), 64, 72
    _, wg, wu, wd, _ = _ffn(1, d, f)
    assert layer.gated_ffn_workspace_bytes(0, d, f, True) == 0
    dw = [torch.full(s, 3.0, device="cuda") for s in ((f, d), (f, d), (d, f))]
    for flags, want in ((256 + 1, 3.0), (256, 0.0)):   # float32 gradients: added to, then written
        rc = lib.pspo_gated_ffn_bwd(None, None, wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), None, 0, d, f, 0, flags, None,
                                    *(t.data_ptr() for t in dw), None, 0, torch.cuda.current_stream().cuda_stream)
        assert rc == 0, lib.pspo_last_error()
        assert all((t == want).all() for t in dw)


@pytest.mark.parametrize("dtype", [BF, F4])
def test_head_norms_at_the_ends_of_float32(dtype):
    """The largest entries whose squares still add up, the first that do not (zeros, as documented), and tiny ones
    (the epsilon alone); the other heads of the token are what they were."""
    N, H, D = 3, 4, 64
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(N, H, D, device="cuda", generator=g).to(dtype)
    x[0, 1], x[1, 2], x[2, 3] = 2.0 ** 60, 2.0 ** 70, 2.0 ** -100
    pos, inv = torch.arange(N, dtype=torch.int32, device="cuda"), torch.ones(16, device="cuda")
    d = torch.ones_like(x)
    y = layer.qk_norm_rope(x, None, None, None, inv, N, positions=pos)["q"]
    b = layer.qk_norm_rope_bwd(d, None, x, None, None, None, inv, N, positions=pos)["dq"]
    z = torch.ones_like(x)
    ref = layer.qk_norm_rope(z, None, None, None, inv, N, positions=pos)["q"]
    # 2^60 and 1 differ by the epsilon in 1 + eps: 5e-7; then one rounding each
    step = (2.0 ** -8 if dtype == BF else 2.0 ** -24) * 2 + 1e-6
    assert ((y[0, 1] - ref[0, 1]).abs() <= step * 1.5).all()
    assert (y[1, 2] == 0).all() and (b[1, 2] == 0).all()
    assert (y[2, 3].abs() <= 2.0 ** -89).all() and torch.isfinite(b[2, 3]).all()   # 2^-100 sqrt(2) / sqrt(eps) < 2^-89
    assert torch.isfinite(y).all() and torch.isfinite(b).all()
