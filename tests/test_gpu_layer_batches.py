"""GPU: head norms and dropout on whole batches, where a wave takes several passes or tokens and the accesses go
past the caches (layer_sizes.py; test_layer_paths_cpu.py holds the sizes against the launch shapes).

Every entry against float64 on the formulas (torch, on the GPU); the tolerances are those derived in
test_gpu_layer_elementwise.py: half a step of the output's type, 4e-6 of a head's largest normed entry (forward),
1e-5 of the gradient's parts (backward), additions in line for the weights' gradients.
"""
import pytest
import torch

from layer_sizes import DROP_PAST, QK_PATHS
from oracle import layer_ops as ol
from paper_2606_29758_amd import layer

pytestmark = pytest.mark.gpu
TYPES = dict(bf16=torch.bfloat16, f32=torch.float32)
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _turn(z, pos, inv, il, back=False):
    if inv is None:
        return z.clone()
    rot = 2 * inv.shape[0]
    ang = pos.double()[:, None, None] * inv.double()
    c, s = torch.cos(ang), torch.sin(ang) * (-1.0 if back else 1.0)
    out = z.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if il else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., a] = z[..., a] * c - z[..., b] * s
    out[..., b] = z[..., a] * s + z[..., b] * c
    return out


def _within(got, want, tol, what):
    e = (got.double() - want).abs()
    assert (e <= tol).all(), (what, float((e - tol).max()), int((e > tol).sum()))


def _side(x, w, pos, inv, il, dtype, y, dout, dx, dw, chain, what):
    """One side (queries or keys): x, y, dout, dx [N, H, D] as the calls took and gave them, against float64."""
    x, w, eps = x.double(), w.double(), 1e-6
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xhat = x * rstd
    z = xhat * w
    ref = _turn(z, pos, inv, il)
    _within(y, ref, STEP[dtype] * ref.abs() + 4e-6 * z.abs().amax(-1, keepdim=True), what + " forward")
    del ref, z
    dz = _turn(dout.double(), pos, inv, il, back=True)
    dzw = dz * w
    ref = rstd * (dzw - xhat * (dzw * xhat).mean(-1, keepdim=True))
    top, xa = dz.abs().amax(-1, keepdim=True), xhat.abs()
    S = rstd * (top * w.abs().max() + xa * (top * w.abs() * xa).mean(-1, keepdim=True))
    _within(dx, ref, STEP[dtype] * ref.abs() + 1e-5 * S, what + " backward")
    _within(dw, (dz * xhat).sum((0, 1)), (chain + 32) * 2.0 ** -24 * (top * xa).sum((0, 1)), what + " weight")


@pytest.mark.parametrize("N,Hq,Hk,D,rot,il,kind", QK_PATHS)
def test_head_norms(N, Hq, Hk, D, rot, il, kind):
    dtype = TYPES[kind]
    g = torch.Generator("cuda").manual_seed(7 * N + 3 * D + Hq)
    new = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    qkv = (new(N, (Hq + Hk) * D + 8) * 1.7).to(dtype)
    q, k = qkv[:, :Hq * D].unflatten(1, (Hq, D)), qkv[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D))
    qw, kw = ((1 + 0.3 * new(D)).to(dtype) for _ in range(2))
    inv = 10000.0 ** (-2.0 * torch.arange(rot // 2, device="cuda") / rot) if rot else None
    pos = torch.randint(0, 200000, (N,), device="cuda", generator=g, dtype=torch.int32)
    dq, dk = new(N, Hq, D).to(dtype), new(N, Hk, D).to(dtype)
    o = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=pos, interleaved=il)
    b = layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, N, positions=pos, interleaved=il)
    per = N // 4096 + 1   # tokens of a wave at most
    # in line: a wave's tokens and its passes, then the lanes', waves' and work-groups' joins
    _side(q, qw, pos, inv, il, dtype, o["q"], dq, b["dq"], b["dq_weight"], per * Hq + 32, "q")
    _side(k, kw, pos, inv, il, dtype, o["k"], dk, b["dk"], b["dk_weight"], per * Hk + 32, "k")


@pytest.mark.parametrize("N,Hq,Hk,D,rot,il,kind", [QK_PATHS[8], QK_PATHS[13], QK_PATHS[22], QK_PATHS[27]])
def test_head_norms_of_a_batch_are_those_of_its_tokens(N, Hq, Hk, D, rot, il, kind):
    """Rotation alone, and with the norm: a token's rows have the same bits in a batch and in a call of 50 tokens."""
    dtype = TYPES[kind]
    g = torch.Generator("cuda").manual_seed(N + D)
    new = lambda *s: torch.randn(*s, device="cuda", generator=g).to(dtype)   # noqa: E731
    q, k, dq, dk = new(N, Hq, D), new(N, Hk, D), new(N, Hq, D), new(N, Hk, D)
    w = new(D)
    inv = 10000.0 ** (-2.0 * torch.arange(rot // 2, device="cuda") / rot)
    pos = torch.randint(0, 200000, (N,), device="cuda", generator=g, dtype=torch.int32)
    for norm in (True, False):
        kw = dict(interleaved=il, norm=norm)
        ws = (w, w) if norm else (None, None)
        o = layer.qk_norm_rope(q, k, *ws, inv, N, positions=pos, **kw)
        b = layer.qk_norm_rope_bwd(dq, dk, q, k, *ws, inv, N, positions=pos, **kw)
        for at in (0, 4093, 4096, 8150, N - 50):
            s = slice(at, at + 50)
            p = layer.qk_norm_rope(q[s], k[s], *ws, inv, 50, positions=pos[s].clone(), **kw)
            r = layer.qk_norm_rope_bwd(dq[s], dk[s], q[s], k[s], *ws, inv, 50, positions=pos[s].clone(), **kw)
            for whole, part in ((o["q"], p["q"]), (o["k"], p["k"]), (b["dq"], r["dq"]), (b["dk"], r["dk"])):
                assert torch.equal(whole[s], part), (norm, at)


@pytest.mark.parametrize("N,Hq,Hk,D,rot,il,kind", [QK_PATHS[8], QK_PATHS[13], QK_PATHS[22], QK_PATHS[27]])
def test_weight_gradients_hold_every_token(N, Hq, Hk, D, rot, il, kind):
    """Terms of one sign (no rotation, positive entries): the sums in float32 are good to `chain` u of themselves, far
    below what one wave's tokens add (1 / 4096)."""
    dtype = TYPES[kind]
    g = torch.Generator("cuda").manual_seed(N + Hq)
    new = lambda *s: (1 + torch.rand(*s, device="cuda", generator=g)).to(dtype)   # noqa: E731
    q, k, w, dq, dk = new(N, Hq, D), new(N, Hk, D), new(D), new(N, Hq, D), new(N, Hk, D)
    b = layer.qk_norm_rope_bwd(dq, dk, q, k, w, w, None, N)
    for x, d, got, H in ((q, dq, b["dq_weight"], Hq), (k, dk, b["dk_weight"], Hk)):
        x = x.double()
        ref = (d.double() * x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)).sum((0, 1))
        chain = (N // 4096 + 1) * H + 32
        _within(got, ref, (chain + 32) * 2.0 ** -24 * ref, "weight")
        assert (chain + 32) * 2.0 ** -24 < 0.25 / 4096


@pytest.mark.parametrize("N,d,kind,to,residual", DROP_PAST)
def test_dropout_past_the_caches(N, d, kind, to, residual):
    """The mask of chosen rows from the oracle's generator, and all rows against calls of 1,000 of them."""
    t, out, p, seed = TYPES[kind], TYPES[to], 0.25, 2 ** 40 + 5
    g = torch.Generator("cuda").manual_seed(N)
    x = (torch.randn(N, d, device="cuda", generator=g) + 3.0).to(t)
    res = torch.randn(N, d, device="cuda", generator=g).to(t) if residual else None
    rows = torch.randperm(3 * N, device="cuda", generator=g)[:N].to(torch.int32)

    def call(s, n):
        ids = rows[s].clone()
        if out == t and (residual or kind == "f32"):
            return layer.dropout_add(x[s], n, p, seed, 9, residual=None if res is None else res[s], row_ids=ids)
        return layer.dropout_bwd(x[s], n, p, seed, 9, row_ids=ids, out_dtype=out)

    y = call(slice(0, N), N)
    at = [0, 1, 255, 15_000, N - 1]
    mask = torch.from_numpy(ol.dropout_mask(rows[at].tolist(), d, p, seed, 9)).cuda()
    part = torch.where(mask, x[at].double() * (65536.0 / ol.keep_threshold(p)), 0.0)
    ref = part if res is None else part + res[at].double()
    size = part.abs() if res is None else part.abs() + res[at].double().abs()
    # the scale and the product 2 u, the sum u; one rounding to the output's type
    _within(y[at], ref, STEP[out] * ref.abs() * (1 + 1e-6) + 3 * 2.0 ** -24 * size, "rows")
    for a in range(0, N, 1000):
        s = slice(a, min(a + 1000, N))
        assert torch.equal(y[s], call(s, s.stop - s.start)), a
