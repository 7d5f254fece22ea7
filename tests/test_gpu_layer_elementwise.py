"""GPU: head norms with rotation, and dropout, against the float64 oracle, through the binding.

Tolerances, from the arithmetic (u = 2^-24):
  * one rounding to the output's type: half a step, 2^-8 (bf16) or 2^-24 (float32) of the value;
  * a turned entry a c - b s of a head whose largest normed entry is m: the sum of squares
    adds at most 8 + 6 terms in line (14 u, halved by the root), root, division and two products
    5 u; the angle's cosine 2 u + pi u, twice; products and sum 3 u: under 32 u, 2e-6 of
    m sqrt(2); 4e-6 m is allowed;
  * its gradient likewise against S = rstd (|dz w|max + |xhat| mean|dz w xhat|), with one more
    sum of 14 terms: 1e-5 S is allowed;
  * a weight's gradient: `chain` additions in line of terms each good to 32 u of max|dz| |xhat|.
"""
import numpy as np
import pytest
import torch

from oracle import layer_ops as ol
from paper_2606_29758_amd import layer, pspo

pytestmark = pytest.mark.gpu
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F4 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _cuda(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def _i32(a):
    return _cuda(np.asarray(a), torch.int32)


def _inputs(N, Hq, Hk, D, rot, dtype, seed, pad=0):
    """q and k as parts of one projection's rows (`pad` further entries a row), weights, frequencies."""
    rng = np.random.default_rng(seed)
    qkv = _cuda(rng.normal(size=(N, (Hq + 2 * Hk) * D + pad)) * np.exp(rng.normal(size=(1, 1))), dtype)
    q = qkv[:, :Hq * D].unflatten(1, (Hq, D))
    k = qkv[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D)) if Hk else None
    qw, kw = (_cuda(1 + 0.3 * rng.normal(size=D), dtype) for _ in range(2))
    inv = _cuda(10000.0 ** (-2.0 * np.arange(rot // 2) / rot), F4) if rot else None
    pos = _i32(rng.integers(0, 200000, N))
    dq = _cuda(rng.normal(size=(N, Hq, D)), dtype)
    dk = _cuda(rng.normal(size=(N, Hk, D)), dtype) if Hk else None
    return q, k, qw, kw, inv, pos, dq, dk


def _check_fwd(got, x, w, pos, inv, eps, il, norm, dtype):
    x, w = _np(x), _np(w)
    inv = np.zeros(0) if inv is None else _np(inv)
    ref = ol.qk_norm_rope(x, w, pos, inv, eps, il, norm)
    z = ol.qk_norm_rope(x, w, pos, np.zeros(0), eps, il, norm)
    m = np.abs(z).max(axis=-1, keepdims=True)
    err = np.abs(_np(got) - ref)
    assert (err <= STEP[dtype] * np.abs(ref) + 4e-6 * m).all(), float((err / (np.abs(ref) + m + 1e-300)).max())


def _check_bwd(dx, dw, dout, x, w, pos, inv, eps, il, norm, dtype, chain):
    x, w, dout = _np(x), _np(w), _np(dout)
    inv = np.zeros(0) if inv is None else _np(inv)
    ref, ref_w = ol.qk_norm_rope_bwd(dout, x, w, pos, inv, eps, il, norm)
    dz = np.abs(ol.rotate(dout, pos, inv, il, back=True)).max(axis=-1, keepdims=True)
    ws = 1.0 if w is None else np.abs(w)
    if norm:
        rstd = 1 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        xh = np.abs(x * rstd)
        S = rstd * (dz * np.max(ws) + xh * np.mean(dz * ws * xh, axis=-1, keepdims=True))
    else:
        S = dz
    err = np.abs(_np(dx) - ref)
    assert (err <= STEP[dtype] * np.abs(ref) + 1e-5 * S).all(), float((err / (np.abs(ref) + S + 1e-300)).max())
    if dw is not None:
        scale = (dz * xh).sum(axis=(0, 1))
        e = np.abs(_np(dw) - ref_w)
        assert (e <= (chain + 32) * 2.0 ** -24 * scale).all(), float((e / (scale + 1e-300)).max())


CASES = [  # N, Hq, Hk, D, rot, interleaved
    (1, 1, 0, 8, 0, False), (1, 28, 4, 128, 128, False), (5, 3, 1, 16, 16, False), (7, 2, 2, 24, 16, True),
    (33, 12, 1, 80, 32, False), (64, 9, 3, 72, 64, False), (63, 5, 2, 96, 96, True), (129, 8, 8, 64, 64, False),
    (17, 4, 2, 256, 64, False), (9, 3, 1, 512, 512, False), (6, 17, 5, 40, 32, True), (3001, 3, 1, 128, 128, False),
]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("N,Hq,Hk,D,rot,il", CASES)
def test_qk_against_the_oracle(N, Hq, Hk, D, rot, il, dtype):
    q, k, qw, kw, inv, pos, dq, dk = _inputs(N, Hq, Hk, D, rot, dtype, 31 * N + D, pad=8)
    p = pos.cpu().numpy()
    o = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=pos, interleaved=il)
    g = layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, N, positions=pos, interleaved=il)
    # in line: a wave's tokens and its passes, then the lanes', waves' and work-groups' joins
    chain = (N // 4096 + 1) * max(Hq, 1) + 6 + 4 + 16 + 6
    for x, w, y, d, dx, dw in ((q, qw, o["q"], dq, g["dq"], g["dq_weight"]), (k, kw, o["k"], dk, g["dk"], g["dk_weight"])):
        if x is None:
            assert y is None and dx is None and (dw == 0).all()   # no keys: their weight's gradient is zero
            continue
        _check_fwd(y, x, w, p, inv, 1e-6, il, True, dtype)
        _check_bwd(dx, dw, d, x, w, p, inv, 1e-6, il, True, dtype, chain)


@pytest.mark.parametrize("il", [False, True])
def test_qk_rotation_only_and_no_weights(il):
    N, Hq, Hk, D, rot = 37, 4, 2, 64, 32
    q, k, qw, kw, inv, pos, dq, dk = _inputs(N, Hq, Hk, D, rot, F4, 5)
    p = pos.cpu().numpy()
    o = layer.qk_norm_rope(q, k, None, None, inv, N, positions=pos, interleaved=il, norm=False)
    g = layer.qk_norm_rope_bwd(dq, dk, q, k, None, None, inv, N, positions=pos, interleaved=il, norm=False)
    _check_fwd(o["q"], q, None, p, inv, 1e-6, il, False, F4)
    _check_bwd(g["dk"], None, dk, k, None, p, inv, 1e-6, il, False, F4, 0)
    assert g["dq_weight"] is None and g["dk_weight"] is None
    assert torch.equal(o["q"][..., rot:], q[..., rot:])   # entries that are not turned pass as they are
    o = layer.qk_norm_rope(q, k, qw, None, inv, N, positions=pos, interleaved=il)
    g = layer.qk_norm_rope_bwd(dq, dk, q, k, qw, None, inv, N, positions=pos, interleaved=il)
    _check_fwd(o["k"], k, None, p, inv, 1e-6, il, True, F4)
    _check_bwd(g["dk"], None, dk, k, None, p, inv, 1e-6, il, True, F4, 0)
    assert g["dk_weight"] is None and g["dq_weight"] is not None


def test_qk_positions_of_packed_prefixes():
    """Positions from the packer's arrays equal the same positions given; empty prefixes; a seq_id out of range."""
    cu = [0, 3, 3, 10, 40, 41]
    N, R = 41, 5
    seq = np.repeat(np.arange(R), np.diff(cu)).astype(np.int32)
    first = [100, 7, 0, 2 ** 30, 5]
    q, k, qw, kw, inv, _, dq, dk = _inputs(N, 4, 2, 64, 64, BF, 9)
    pos = ol.positions(seq, cu, first, N)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    at = dict(seq_id=_i32(seq), cu_seqlens=_i32(cu), first_pos=_i32(first), err_flag=err)
    a = layer.qk_norm_rope(q, k, qw, kw, inv, N, **at)
    b = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=_i32(pos))
    assert torch.equal(a["q"], b["q"]) and torch.equal(a["k"], b["k"]) and int(err) == 0
    _check_fwd(a["q"], q, qw, pos, inv, 1e-6, False, True, BF)
    c = layer.qk_norm_rope(q, k, qw, kw, inv, N, seq_id=at["seq_id"], cu_seqlens=at["cu_seqlens"])
    _check_fwd(c["q"], q, qw, ol.positions(seq, cu, None, N), inv, 1e-6, False, True, BF)
    seq[4], seq[20] = R, -1
    at["seq_id"] = _i32(seq)
    a = layer.qk_norm_rope(q, k, qw, kw, inv, N, **at)
    assert int(err) == pspo.DEVERR_SEQ_ID
    _check_fwd(a["q"], q, qw, ol.positions(seq, cu, first, N), inv, 1e-6, False, True, BF)
    err.zero_()
    layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, N, **at)
    assert int(err) == pspo.DEVERR_SEQ_ID


def test_qk_far_positions():
    """The whole int32 range: the angle is formed in float64."""
    p = np.array([0, 1, -1, 65536, 10 ** 6, 2 ** 31 - 1, -2 ** 31], dtype=np.int64)
    q, k, qw, kw, inv, _, _, _ = _inputs(len(p), 2, 1, 32, 32, F4, 12)
    o = layer.qk_norm_rope(q, k, qw, kw, inv, len(p), positions=_i32(p))
    # turns up to 3.4e8 carry 2^-53 each: 1e-7 turns at most, 6e-7 of the entry's pair
    _check_fwd(o["q"], q, qw, p, inv, 1e-6, False, True, F4)


def test_qk_rows_behind_and_values_that_are_not_finite():
    N, cap, D = 10, 16, 64
    q, k, qw, kw, inv, pos, dq, dk = _inputs(cap, 3, 1, D, 32, F4, 13)
    ref = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=pos)
    q, k = q.clone(), k.clone()
    q[10:] = float("nan")                      # rows behind the N-th are not read
    q[2, 1] = float("inf")                     # one head of one token
    q[3, 0, 5] = float("nan")
    q[4, 2] = 0.0
    qo, ko = torch.full((cap, 3, D), 7.0, device="cuda"), torch.full((cap, 1, D), 7.0, device="cuda")
    o = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=pos, q_out=qo, k_out=ko)
    assert (qo[N:] == 7).all() and (ko[N:] == 7).all()
    same = torch.ones(N, 3, dtype=torch.bool)
    same[2, 1] = same[3, 0] = same[4, 2] = False
    assert torch.equal(o["q"].cpu()[same], ref["q"].cpu()[same]) and torch.equal(o["k"], ref["k"])
    assert torch.isnan(o["q"][3, 0]).all() and (o["q"][4, 2] == 0).all()
    g = layer.qk_norm_rope_bwd(dq, dk, torch.zeros_like(q), k, qw, kw, inv, N, positions=pos)
    assert torch.isfinite(g["dq"]).all() and (g["dq_weight"] == 0).all()   # a head of zeros: 1 / sqrt(eps)


def test_qk_no_tokens():
    q, k, qw, kw, inv, pos, dq, dk = _inputs(2, 3, 1, 64, 32, BF, 14)
    o = layer.qk_norm_rope(q, k, qw, kw, inv, 0, positions=pos)
    assert o["q"].shape == (0, 3, 64)
    g = layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, 0, positions=pos)
    assert (g["dq_weight"] == 0).all() and (g["dk_weight"] == 0).all()


def test_qk_offsets_past_32_bits():
    """Rows 65,536 entries apart: the last rows lie past 2^32 bytes."""
    N, D, stride = 40000, 128, 65536
    big = torch.empty(N * stride, dtype=BF, device="cuda")
    q = big.as_strided((N, 1, D), (stride, D, 1))
    q.copy_(torch.randn(N, 1, D, device="cuda", generator=torch.Generator("cuda").manual_seed(1)))
    w = torch.ones(D, dtype=BF, device="cuda")
    inv = _cuda(10000.0 ** (-np.arange(64) / 64), F4)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    a = layer.qk_norm_rope(q, None, w, None, inv, N, positions=pos)["q"]
    b = layer.qk_norm_rope(q.contiguous(), None, w, None, inv, N, positions=pos)["q"]
    assert torch.equal(a, b)
    at = slice(N - 20, N)
    _check_fwd(a[at], q[at], w, pos[at].cpu().numpy(), inv, 1e-6, False, True, BF)


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

def _check_drop(got, x, res, mask, p, dtype):
    x, res = _np(x), _np(res)
    ref = ol.dropout_add(x, res, mask, p)
    # the scale and the product 2 u of |x| scale, the sum u: 3 u of the parts' sizes
    parts = np.abs(ref if res is None else np.abs(res) + np.abs(ref - res))
    err = np.abs(_np(got) - ref)
    assert (err <= STEP[dtype] * np.abs(ref) * (1 + 1e-6) + 3 * 2.0 ** -24 * parts).all()


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("N,d,p,seed,offset", [
    (1, 8, 0.5, 0, 0), (3, 16, 0.1, 2 ** 63 + 11, 2 ** 40 + 3), (5, 24, 0.25, 7, 1), (9, 72, 0.9, 1, 0),
    (33, 136, 0.05, 3, 9), (2, 520, 0.5, 4, 2 ** 64 - 1), (13, 3584, 0.1, 5, 6), (1, 8200, 0.3, 6, 0),
    (4, 64, 0.0, 8, 0), (6, 64, 0.9999999, 8, 0), (257, 32, 0.5, 9, 0)])
def test_dropout_against_the_oracle(N, d, p, seed, offset, dtype):
    rng = np.random.default_rng(N + d)
    x, res = _cuda(rng.normal(size=(N, d)) + 3.0, dtype), _cuda(rng.normal(size=(N, d)), dtype)
    mask = ol.dropout_mask(range(N), d, p, seed, offset)
    y = layer.dropout_add(x, N, p, seed, offset)
    assert np.array_equal(_np(y) != 0, mask)      # every input is away from zero
    _check_drop(y, x, None, mask, p, dtype)
    _check_drop(layer.dropout_add(x, N, p, seed, offset, residual=res), x, res, mask, p, dtype)
    for out in (BF, F4):
        dx = layer.dropout_bwd(x, N, p, seed, offset, out_dtype=out)
        assert dx.dtype == out
        _check_drop(dx, x, None, mask, p, out)
    if p == 0.0:
        assert torch.equal(y, x)


def test_dropout_gradient_is_the_difference():
    """sum(y dy) along a direction v: linear in x, so one difference of float32 steps is exact up to rounding."""
    N, d, p = 17, 256, 0.3
    g = torch.Generator("cuda").manual_seed(3)
    x, v, dy = (torch.randn(N, d, device="cuda", generator=g) for _ in range(3))
    dx = layer.dropout_bwd(dy, N, p, 99)
    up, down = (layer.dropout_add(x + s * v, N, p, 99).double() for s in (0.5, -0.5))
    diff = ((up - down) * dy.double()).sum()
    got = (dx.double() * v.double()).sum()
    # both sides' terms carry some 4 roundings of |y| |dy|
    bound = 8 * 2.0 ** -24 * ((up.abs() + down.abs() + (x.abs() + v.abs()).double() / 0.7) * dy.double().abs()).sum()
    assert abs(float(diff - got)) <= float(bound)


def test_dropout_masks_follow_the_source_rows():
    """The packer's src_row as row ids: a kept token's mask does not depend on the draw of the cutoffs."""
    N, d = 50, 64
    x = torch.ones(N, d, device="cuda")
    full = layer.dropout_add(x, N, 0.5, 21, 4)
    rows = torch.tensor([3, 4, 5, 20, 21, 49], dtype=torch.int32, device="cuda")
    part = layer.dropout_add(x, len(rows), 0.5, 21, 4, row_ids=rows)
    assert torch.equal(part, full[rows.long()])
    same = layer.dropout_add(x, 2, 0.5, 21, 4, row_ids=_i32([7, 7]))
    assert torch.equal(same[0], same[1])
    neg = layer.dropout_add(x, 1, 0.5, 21, 4, row_ids=_i32([-1]))
    assert np.array_equal(_np(neg) != 0, ol.dropout_mask([2 ** 32 - 1], d, 0.5, 21, 4))
    assert not torch.equal(full, layer.dropout_add(x, N, 0.5, 21, 5))
    assert not torch.equal(full, layer.dropout_add(x, N, 0.5, 22, 4))


def test_dropout_rows_behind_and_values_that_are_not_finite():
    N, cap, d, p = 5, 9, 40, 0.5
    x = torch.ones(cap, d, dtype=BF, device="cuda")
    x[1] = float("nan")
    x[2] = float("inf")
    out = torch.full((cap, d), 3.0, dtype=BF, device="cuda")
    y = layer.dropout_add(x, N, p, 1, out=out)
    m = torch.from_numpy(ol.dropout_mask(range(N), d, p, 1, 0))
    assert (out[N:] == 3).all()
    assert (y.cpu()[~m] == 0).all()               # a dropped NaN or Inf leaves nothing
    assert torch.isnan(y.cpu()[1][m[1]]).all() and torch.isinf(y.cpu()[2][m[2]]).all()
    assert layer.dropout_add(x, 0, p, 1).shape == (0, d)
    assert layer.dropout_bwd(x, 0, p, 1).shape == (0, d)


def test_dropout_past_32_bits():
    """More than 2^31 entries (past 2^32 bytes): the last rows against the oracle, the middle against small calls."""
    N, d, p = 600_011, 3584, 0.25
    x = torch.ones(N, d, dtype=BF, device="cuda")
    y = layer.dropout_add(x, N, p, 5, 6, residual=x)
    at = [0, 299_593, 299_594, N - 1]             # 2^30 entries lie between the second and the third
    mask = ol.dropout_mask(at, d, p, 5, 6)
    for i, n in enumerate(at):
        _check_drop(y[n:n + 1], x[n:n + 1], x[n:n + 1], mask[i:i + 1], p, BF)


# ---------------------------------------------------------------------------
# both: refusals, streams, graphs
# ---------------------------------------------------------------------------

def test_refusals_of_device_tensors():
    x = torch.ones(8, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError, match="overlaps"):
        layer.dropout_add(x, 8, 0.1, 1, out=x)
    with pytest.raises(ValueError, match="contiguous"):
        layer.dropout_add(x.t(), 8, 0.1, 1)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        layer.dropout_add(x.half(), 8, 0.1, 1)
    with pytest.raises(ValueError, match="residual"):
        layer.dropout_add(x, 8, 0.1, 1, residual=x[:4])
    with pytest.raises(ValueError, match="row_ids"):
        layer.dropout_add(x, 8, 0.1, 1, row_ids=_i32([1, 2]))
    with pytest.raises(pspo.PspoError, match="p must lie"):
        layer.dropout_add(x, 8, 1.0, 1)
    with pytest.raises(pspo.PspoError, match="p must lie"):
        layer.dropout_add(x, 8, float("nan"), 1)
    with pytest.raises(pspo.PspoError, match="misaligned"):
        layer.dropout_add(torch.ones(8 * 64 + 1, dtype=BF, device="cuda")[1:].view(8, 64), 8, 0.1, 1)
    with pytest.raises(pspo.PspoError, match="d % 8"):
        layer.dropout_add(torch.ones(8, 12, dtype=BF, device="cuda"), 8, 0.1, 1)
    q, k, qw, kw, inv, pos, dq, dk = _inputs(8, 2, 1, 64, 32, BF, 1)
    with pytest.raises(ValueError, match="must be given"):
        layer.qk_norm_rope(q, k, qw, kw, inv, 8)
    with pytest.raises(ValueError, match="fewer than N"):
        layer.qk_norm_rope(q, k, qw, kw, inv, 9, positions=pos)
    with pytest.raises(ValueError, match="contiguous"):
        layer.qk_norm_rope(q.transpose(1, 2), k, qw, kw, inv, 8, positions=pos)
    with pytest.raises(pspo.PspoError, match="16-byte"):
        layer.qk_norm_rope(torch.ones(8 * 132, dtype=BF, device="cuda").as_strided((8, 2, 64), (132, 64, 1)), None, qw,
                           None, inv, 8, positions=pos)
    with pytest.raises(pspo.PspoError, match="strides"):
        layer.qk_norm_rope(qw.as_strided((8, 1, 64), (0, 64, 1)), None, qw, None, inv, 8, positions=pos)
    with pytest.raises(pspo.PspoError, match="rot_dim"):
        layer.qk_norm_rope(q, k, qw, kw, inv[:12], 8, positions=pos)
    with pytest.raises(pspo.PspoError, match="eps"):
        layer.qk_norm_rope(q, k, qw, kw, inv, 8, positions=pos, eps=0.0)
    with pytest.raises(pspo.PspoError, match="weights need"):
        layer.qk_norm_rope(q, k, qw, kw, inv, 8, positions=pos, norm=False)
    with pytest.raises(pspo.PspoError, match="workspace"):
        layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, 8, positions=pos,
                               workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


def test_streams_and_graph_replays():
    """The calls on a stream of their own, and captured and replayed on new inputs, give the eager bits."""
    N, D = 700, 128
    q, k, qw, kw, inv, pos, dq, dk = _inputs(N, 6, 2, D, 128, BF, 77)
    x = torch.randn(N, 512, device="cuda", dtype=F4)

    def calls():
        a = layer.qk_norm_rope(q, k, qw, kw, inv, N, positions=pos)
        b = layer.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, inv, N, positions=pos)
        y = layer.dropout_add(x, N, 0.1, 5, 1, residual=x)
        return [a["q"], a["k"], b["dq"], b["dk"], b["dq_weight"], b["dk_weight"], y,
                layer.dropout_bwd(y, N, 0.1, 5, 1, out_dtype=BF)]

    ref = [t.clone() for t in calls()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = calls()
    for step in range(3):
        q.mul_(-1.0 if step else 1.0)
        x.add_(1.0)
        want = [t.clone() for t in calls()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), step
