"""GPU: the run of test_gpu_layer_run.py, each call against float64 on the inputs that it was given.

The whole run is held by a bound that lets twelve roundings pile up; here every stage starts from the tensors that
the stage before it gave, so that a call that is a few per cent off, or takes the wrong one of two tensors, shows.
Tolerance, in relative 2-norm: a rounding to bf16 is off by 2^-8 / sqrt(3) rms at most.  One rounding stands in the
norms, dropout and their gradients: 2^-8 is allowed; two in the feed-forward block and its gradients, sqrt(2/3) 2^-8:
2^-7; none in the norms' weight gradients and the float32 dropout: 2^-16 (sums of some thousand terms); the loss call
rounds the logit gradient once: 2^-8.
"""
import numpy as np
import pytest
import torch

import test_gpu_layer_run as run
from oracle import layer_ops as ol
from paper_2606_29758_amd import layer

from parity_util import f32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
ONE, TWO, SUMS = 2.0 ** -8, 2.0 ** -7, 2.0 ** -16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, tol, what):
    got = _np(got)
    assert got.shape == want.shape, what
    e = np.linalg.norm(got - want) / np.linalg.norm(want)
    print(f"  {what}: {e:.2e}", flush=True)
    assert e <= tol, (what, e)


def test_every_stage_of_the_run():
    s = run._setup()
    pk, N = run._pack(s, seed=0)
    qkv, q, k, at, o, h1, ffn, h2, loss = run._forward(s, pk, N)
    rows = pk["src_row"][:N].cpu().numpy()
    pos = ol.positions(pk["seq_id"][:N].cpu().numpy(), pk["cu_seqlens"].cpu().numpy(), s["first"].cpu().numpy(), N)
    inv = _np(s["inv"])
    m1, m2 = (ol.dropout_mask(rows, run.D_MODEL, run.DROP, run.SEED, run.OFFSET + i) for i in (0, 1))
    for name, x, w in (("q", q, s["qw"]), ("k", k, s["kw"])):
        _near(o[name], ol.qk_norm_rope(_np(x[:N]), _np(w), pos, inv, 1e-6), ONE, name)
    mix = run._mix(o["q"].float(), o["k"].float()).to(BF)
    _near(h1, ol.dropout_add(_np(mix), _np(pk["hidden"][:N]), m1, run.DROP), ONE, "first sum")
    weights = [_np(s[n]) for n in ("wg", "wu", "wd")]
    y, pre = ol.gated_ffn(_np(h1), *weights, "silu")
    _near(ffn["y"], y, TWO, "block")
    _near(ffn["preact"], pre, SUMS, "pre-activations")
    _near(h2, ol.dropout_add(_np(ffn["y"]), _np(h1), m2, run.DROP), ONE, "second sum")

    # the loss call on these rows, by autograd in float64
    h = h2.double().cpu().requires_grad_()
    head = s["head"].double().cpu().requires_grad_()
    logp = torch.log_softmax(h @ head.T, -1)[torch.arange(N), pk["target"][:N].long().cpu()]
    rho = torch.exp(logp - pk["logp_old"][:N].double().cpu())
    adv = s["adv"].double().cpu()[pk["seq_id"][:N].long().cpu()]
    sur = torch.minimum(rho * adv, rho.clamp(1 - f32(0.1), 1 + f32(0.1)) * adv)
    (-(f32(1.0 / s["R"]) * pk["weight"][:N].double().cpu() * sur).sum()).backward()
    _near(loss["d_hidden"][:N], h.grad.numpy(), ONE, "d_hidden")
    _near(loss["d_w_head"], head.grad.numpy(), ONE, "d_w_head")

    dh2 = loss["d_hidden"][:N]
    scale = 65536.0 / ol.keep_threshold(run.DROP)
    dy = layer.dropout_bwd(dh2, N, run.DROP, run.SEED, run.OFFSET + 1, row_ids=pk["src_row"], out_dtype=BF)
    _near(dy, np.where(m2, _np(dh2) * scale, 0.0), ONE, "dy")
    dy32 = layer.dropout_bwd(dh2, N, run.DROP, run.SEED, run.OFFSET + 1, row_ids=pk["src_row"])
    _near(dy32, np.where(m2, _np(dh2) * scale, 0.0), SUMS, "dy in float32")
    b = layer.gated_ffn_bwd(dy, h1, s["wg"], s["wu"], s["wd"], N, preact=ffn["preact"])
    for name, want in zip(("dx", "dw_gate", "dw_up", "dw_down"), ol.gated_ffn_bwd(_np(dy), _np(h1), *weights, "silu")):
        _near(b[name], want, TWO, name)
    dh1 = dh2 + b["dx"].float()
    dmix = layer.dropout_bwd(dh1, N, run.DROP, run.SEED, run.OFFSET, row_ids=pk["src_row"], out_dtype=BF)
    _near(dmix, np.where(m1, _np(dh1) * scale, 0.0), ONE, "dmix")
    dm = dmix.float().view(N, run.HQ, run.HD)
    dq_o = (dm * o["k"].float().repeat_interleave(run.HQ // run.HK, dim=1)).to(BF)
    dk_o = (dm * o["q"].float()).view(N, run.HK, run.HQ // run.HK, run.HD).sum(2).to(BF)
    g = layer.qk_norm_rope_bwd(dq_o, dk_o, q, k, s["qw"], s["kw"], s["inv"], N, **at)
    for name, x, w, d in (("q", q, s["qw"], dq_o), ("k", k, s["kw"], dk_o)):
        dx, dw = ol.qk_norm_rope_bwd(_np(d), _np(x[:N]), _np(w), pos, inv, 1e-6)
        _near(g["d" + name], dx, ONE, "d" + name)
        _near(g[f"d{name}_weight"], dw, SUMS, f"d{name}_weight")
    # and the run's own backward gave the same
    whole = run._backward(s, pk, N, (qkv, q, k, at, o, h1, ffn, h2, loss))
    assert torch.equal(whole["dq"], g["dq"]) and torch.equal(whole["dk"], g["dk"])
    assert all(torch.equal(whole[a], b[c]) for a, c in (("wg", "dw_gate"), ("wu", "dw_up"), ("wd", "dw_down")))
