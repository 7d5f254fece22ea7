"""GPU: the layer operators together, as a policy's update uses them on the packer's output.

Packed prefixes -> head norms with rotation at the packed positions -> a token-wise mixing of the
turned heads -> dropout by source row with the residual sum -> gated feed-forward block -> dropout
with the residual sum -> the LM-head PPO loss, and back through all of it with the calls' own
backward passes.  The reference is torch's autograd in float64 on the formulas, with the masks from
the oracle's generator.  (Attention itself is not this library's: the mixing stands in its place,
and its gradient is torch's, in float32.)

Tolerance: in relative 2-norm, each rounding of a tensor to bf16 costs at most half a step, 2^-8.
The forward rounds q, k, the first sum, h, y, the second sum; the backward the loss's gradient,
dg / du, the block's dx, two dropout gradients, dq / dk: 12 steps, 12 * 2^-8 = 4.7e-2 at most if
all point one way and no factor amplifies; the products' operands are independent draws, so they
do not.
"""
import numpy as np
import pytest
import torch

from oracle import layer_ops as ol
from paper_2606_29758_amd import layer, pspo

from parity_util import f32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
REL = 12 * 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    layer.load()


def _rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


P, K, D_MODEL, F, V, HQ, HK, HD, DROP, SEED, OFFSET = 3, 2, 256, 520, 1024, 4, 2, 64, 0.1, 77, 3


def _setup():
    g = torch.Generator("cuda").manual_seed(5)
    rng = np.random.default_rng(5)
    R = P * K
    lengths = rng.integers(20, 60, R).astype(np.int32)
    xi, off = [], [0]
    for p in range(P):
        T = int(lengths[p * K:(p + 1) * K].max())
        xi.append(np.minimum.accumulate(np.linspace(1.0, 0.3, T)))
        off.append(off[-1] + T)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)   # noqa: E731
    S = int(lengths.sum())
    new = lambda *s, k=1.0: (torch.randn(*s, device="cuda", generator=g) * k).to(BF)   # noqa: E731
    s = dict(lengths=dev(lengths, torch.int32), xi=dev(np.concatenate(xi), torch.float64), off=dev(off, torch.int64),
             target=torch.randint(0, V, (S,), device="cuda", generator=g, dtype=torch.int32), S=S, R=R,
             first=dev(rng.integers(0, 500, R), torch.int32), hidden=new(S, D_MODEL),
             logp_old=torch.full((S,), -np.log(V), device="cuda") + 0.05 * torch.randn(S, device="cuda", generator=g),
             adv=dev(rng.normal(size=R), torch.float32), head=new(V, D_MODEL, k=0.02),
             qkv=new(D_MODEL, (HQ + 2 * HK) * HD, k=1 / 16), qw=(1 + 0.2 * new(HD).float()).to(BF),
             kw=(1 + 0.2 * new(HD).float()).to(BF), wg=new(F, D_MODEL, k=1 / 16), wu=new(F, D_MODEL, k=1 / 16),
             wd=new(D_MODEL, F, k=1 / 23),
             inv=dev(10000.0 ** (-np.arange(HD // 2) / (HD // 2)), torch.float32))
    return s


def _mix(q, k):
    """A token's queries times its keys, head by head of the group: [N, HQ * HD]."""
    return (q * k.repeat_interleave(HQ // HK, dim=1)).reshape(q.shape[0], -1)


def _pack(s, seed):
    cut = pspo.sample_cutoffs(s["xi"], s["off"], s["lengths"], P, K, seed)
    pk = pspo.pack_prefixes(cut, s["lengths"], s["xi"], s["off"], P, K, s["S"], target_full=s["target"],
                            logp_old_full=s["logp_old"], hidden_full=s["hidden"])
    return pk, int(pk["n_tokens"])


def _forward(s, pk, N):
    qkv = (pk["hidden"].float() @ s["qkv"].float()).to(BF)        # every row of the capacity: a strided view below
    q, k = qkv[:, :HQ * HD].unflatten(1, (HQ, HD)), qkv[:, HQ * HD:(HQ + HK) * HD].unflatten(1, (HK, HD))
    at = dict(seq_id=pk["seq_id"], cu_seqlens=pk["cu_seqlens"], first_pos=s["first"])
    o = layer.qk_norm_rope(q, k, s["qw"], s["kw"], s["inv"], N, **at)
    mix = _mix(o["q"].float(), o["k"].float()).to(BF)
    h1 = layer.dropout_add(mix, N, DROP, SEED, OFFSET, residual=pk["hidden"], row_ids=pk["src_row"])
    ffn = layer.gated_ffn(h1, s["wg"], s["wu"], s["wd"], N, keep=True)
    h2 = layer.dropout_add(ffn["y"], N, DROP, SEED, OFFSET + 1, residual=h1, row_ids=pk["src_row"])
    loss = pspo.loss_fwd_bwd(h2, s["head"], pk["target"], pk["logp_old"], pk["weight"], pk["seq_id"], s["adv"], N, 0.1, 0.1,
                             1.0 / (P * K))
    return qkv, q, k, at, o, h1, ffn, h2, loss


def _backward(s, pk, N, fwd):
    qkv, q, k, at, o, h1, ffn, h2, loss = fwd
    dh2 = loss["d_hidden"]                                          # float32, straight into the dropout's backward
    dy = layer.dropout_bwd(dh2, N, DROP, SEED, OFFSET + 1, row_ids=pk["src_row"], out_dtype=BF)
    b = layer.gated_ffn_bwd(dy, h1, s["wg"], s["wu"], s["wd"], N, preact=ffn["preact"])
    dh1 = dh2 + b["dx"].float()
    dmix = layer.dropout_bwd(dh1, N, DROP, SEED, OFFSET, row_ids=pk["src_row"], out_dtype=BF).float()
    dm = dmix.view(N, HQ, HD)
    kk = o["k"].float().repeat_interleave(HQ // HK, dim=1)
    dq_o = (dm * kk).to(BF)
    dk_o = (dm * o["q"].float()).view(N, HK, HQ // HK, HD).sum(2).to(BF)   # shared key heads: their group's sum
    qk = layer.qk_norm_rope_bwd(dq_o, dk_o, q, k, s["qw"], s["kw"], s["inv"], N, **at)
    return dict(dq=qk["dq"], dk=qk["dk"], qw=qk["dq_weight"], kw=qk["dk_weight"], wg=b["dw_gate"], wu=b["dw_up"],
                wd=b["dw_down"], head=loss["d_w_head"], h0=dh1)


def _reference(s, pk, N, qkv):
    """Loss and gradients by autograd in float64."""
    d = lambda t: t.detach().double().cpu()   # noqa: E731
    leaf = {n: d(s[n]).requires_grad_() for n in ("qw", "kw", "wg", "wu", "wd", "head")}
    x = d(qkv[:N])
    q = x[:, :HQ * HD].unflatten(1, (HQ, HD)).clone().requires_grad_()
    k = x[:, HQ * HD:(HQ + HK) * HD].unflatten(1, (HK, HD)).clone().requires_grad_()
    h0 = d(pk["hidden"][:N]).requires_grad_()
    seq, cu = pk["seq_id"][:N].cpu().numpy(), pk["cu_seqlens"].cpu().numpy()
    pos = torch.from_numpy(ol.positions(seq, cu, s["first"].cpu().numpy(), N)).double()
    ang = pos[:, None] * d(s["inv"])[None]
    cos, sin = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def turned(t, w):
        z = w * t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)
        a, b = z[..., :HD // 2], z[..., HD // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    rows = pk["src_row"][:N].cpu().numpy()
    scale = 65536.0 / ol.keep_threshold(DROP)
    drop = lambda t, o: t * torch.from_numpy(ol.dropout_mask(rows, t.shape[1], DROP, SEED, o)).double() * scale   # noqa: E731
    h1 = h0 + drop(_mix(turned(q, leaf["qw"]), turned(k, leaf["kw"])), OFFSET)
    y = (torch.nn.functional.silu(h1 @ leaf["wg"].T) * (h1 @ leaf["wu"].T)) @ leaf["wd"].T
    h2 = h1 + drop(y, OFFSET + 1)
    logp = torch.log_softmax(h2 @ leaf["head"].T, -1)[torch.arange(N), pk["target"][:N].long().cpu()]
    rho = torch.exp(logp - d(pk["logp_old"][:N]))
    adv = d(s["adv"])[torch.from_numpy(seq).long()]
    sur = torch.minimum(rho * adv, rho.clamp(1 - f32(0.1), 1 + f32(0.1)) * adv)
    loss = -(f32(1.0 / (P * K)) * d(pk["weight"][:N]) * sur).sum()
    loss.backward()
    return float(loss.detach()), dict({n: t.grad for n, t in leaf.items()}, dq=q.grad, dk=k.grad, h0=h0.grad), rho.detach()


def test_layer_run_against_autograd():
    s = _setup()
    pk, N = _pack(s, seed=0)
    fwd = _forward(s, pk, N)
    got = _backward(s, pk, N, fwd)
    want_loss, want, rho = _reference(s, pk, N, fwd[0])
    # the run's rounded states move the ratios: tokens that sit on a clip bound may fall on its other side
    near = int(((rho - 1.1).abs() < 5e-3).sum() + ((rho - 0.9).abs() < 5e-3).sum())
    print(f"[layer run] N = {N} of {s['S']}, loss {float(fwd[-1]['loss']):.6e} / {want_loss:.6e}, {near} near the clip",
          flush=True)
    extra = near / N
    assert abs(float(fwd[-1]["loss"]) - want_loss) <= REL * abs(want_loss) + 1e-3
    for n, w in want.items():
        e = _rel(got[n].cpu(), w)
        print(f"  {n}: {e:.2e}", flush=True)
        assert e <= REL + extra, n


def test_kept_tokens_do_not_depend_on_the_draw():
    """Two draws of the cutoffs: the tokens that both keep have the same states, bit for bit."""
    s = _setup()
    seen = {}
    for seed in (0, 1):
        pk, N = _pack(s, seed)
        h2 = _forward(s, pk, N)[7]
        for i, r in enumerate(pk["src_row"][:N].tolist()):
            if r in seen and seen[r][0] != seed:
                assert torch.equal(seen[r][1], h2[i]), r
            seen[r] = (seed, h2[i])
    assert len(seen) > 50


def test_layer_run_captured():
    """The whole run, forward and backward, captured into a graph and replayed between eager passes on new inputs."""
    s = _setup()
    pk, N = _pack(s, seed=0)

    def run():
        f = _forward(s, pk, N)
        b = _backward(s, pk, N, f)
        return [f[7], f[8]["loss"], *b.values()]

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for step in range(3):
        pk["hidden"].mul_(-1.0 if step else 1.0)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), step
