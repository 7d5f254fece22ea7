"""GPU: the objectives together, as an update uses them on the packer's output.

Packed prefixes -> a gated feed-forward block -> the reference's log-probs under another head (the score proxy's call)
-> the policy loss with its penalty, a preference loss over pairs of the same completions and distillation from the
lists that a rollout reports, all three adding to one float32 head gradient -> their sum back through the block.  The
reference is torch's autograd in float64 on the formulas.

Tolerance, in relative 2-norm (half a bf16 step is 2^-8 relative): the forward rounds h and y; the losses' gradients of
y take the softmax entries and a result each, of up to three terms that may partly cancel (the sum of their norms is
what counts); the block's backward rounds dg, du and its results.  Head gradient: softmax entries and scaled rows, of
rows of y that are themselves off by 2 * 2^-8.
"""
import numpy as np
import pytest
import torch

from paper_2606_29758_amd import layer, objective, pspo, synth

pytestmark = pytest.mark.gpu
BF, STEP = torch.bfloat16, 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


def _cuda(a, t):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)


@pytest.fixture(scope="module")
def batch():
    """The tiny workload: packed prefixes, lists of 16, a reference head near the policy's."""
    wl = synth.make_workload("tiny")
    cfg = wl.cfg
    hidden = _cuda(wl.hidden_bits.view(np.int16), torch.int16).view(BF)
    head = _cuda(wl.w_bits.view(np.int16), torch.int16).view(BF)
    g = torch.Generator("cuda").manual_seed(3)
    new = lambda *s, k=1.0: (torch.randn(*s, device="cuda", generator=g) * k).to(BF)   # noqa: E731
    d, f = cfg.d, 264
    ids, logp = synth.make_topk(wl)
    b = dict(wl=wl, cfg=cfg, hidden=hidden, head=head, wg=new(f, d, k=d ** -0.5), wu=new(f, d, k=d ** -0.5),
             wd=new(d, f, k=f ** -0.5), ids=_cuda(ids, torch.int32), topk=_cuda(logp, torch.float32),
             adv=_cuda(wl.advantage, torch.float32), target=_cuda(wl.target_full, torch.int32))
    b["ref_head"] = (head.float() + 0.004 * torch.randn(head.shape, device="cuda", generator=g)).to(BF)
    return b


def _pack(b, seed):
    wl, cfg = b["wl"], b["cfg"]
    lengths, xi, off = _cuda(wl.lengths, torch.int32), _cuda(wl.xi, torch.float64), _cuda(wl.xi_off, torch.int64)
    cut = pspo.sample_cutoffs(xi, off, lengths, cfg.P, cfg.K, seed)
    pk = pspo.pack_prefixes(cut, lengths, xi, off, cfg.P, cfg.K, int(wl.total_tokens), target_full=b["target"],
                            hidden_full=b["hidden"])
    return pk, int(pk["n_tokens"])


PAIRS = ([0, 1, 4, 6], [3, 2, 5, 7])
EPS, COEF, T, BETA = 0.2, 0.1, 2.0, 0.1


def _run(b, pk, N, grads=None):
    """The calls of one update; grads: the buffers to reuse."""
    cfg = b["cfg"]
    x = pk["hidden"]
    ffn = layer.gated_ffn(x, b["wg"], b["wu"], b["wd"], N, keep=True)
    y = ffn["y"]
    ref = pspo.score_proxy(y, b["ref_head"], pk["target"], N)["logp"]
    old = (ref - 0.01).contiguous()
    dw = torch.zeros(cfg.V, cfg.d, device="cuda")
    chosen, rejected = (torch.tensor(p, dtype=torch.int32, device="cuda") for p in PAIRS)
    rows = pk["src_row"][:N].long()
    kw = dict(d_w_head=dw, accumulate=True)
    o = [objective.policy_loss(y, b["head"], pk["target"], old, pk["weight"], pk["seq_id"], b["adv"], N, EPS, EPS, 1.0 / N,
                               logp_ref=ref, kl_coef=COEF, d_hidden=torch.empty(N, cfg.d, device="cuda"), **kw),
         objective.preference_loss(y, b["head"], pk["target"], pk["cu_seqlens"], chosen, rejected, N, BETA, 0.25,
                                   logp_ref=ref, d_hidden=torch.empty(N, cfg.d, device="cuda"), **kw),
         objective.distill_loss(y, b["head"], b["ids"][rows].contiguous(), b["topk"][rows].contiguous(), N, 1.0 / N,
                                weight=pk["weight"], temperature=T, d_hidden=torch.empty(N, cfg.d, device="cuda"), **kw)]
    dy = (o[0]["d_hidden"] + o[1]["d_hidden"] + o[2]["d_hidden"]).to(BF)
    g = layer.gated_ffn_bwd(dy, x, b["wg"], b["wu"], b["wd"], N, preact=ffn["preact"])
    return dict(y=y, ref=ref, old=old, o=o, dw=dw, dy=dy, g=g)


def _want(b, pk, N, r):
    """The same in float64, by autograd."""
    D = lambda t: t.detach().double()   # noqa: E731
    x = D(pk["hidden"][:N])
    p = {n: D(b[n]).requires_grad_() for n in ("wg", "wu", "wd", "head")}
    x.requires_grad_()
    y = (torch.nn.functional.silu(x @ p["wg"].T) * (x @ p["wu"].T)) @ p["wd"].T
    z = y @ p["head"].T
    i = torch.arange(N, device="cuda")
    target, seq, c = pk["target"][:N].long(), pk["seq_id"][:N].long(), D(pk["weight"][:N])
    l = torch.log_softmax(z, 1)[i, target]
    ref, old, A = D(r["ref"]), D(r["old"]), D(b["adv"])[seq]
    rho = torch.exp(l - old)
    u = l - ref
    policy = (c * (COEF * (torch.exp(-u) - 1 + u) - torch.minimum(rho * A, rho.clamp(1 - EPS, 1 + EPS) * A))).sum() / N
    ratio = torch.zeros(b["cfg"].P * b["cfg"].K, dtype=torch.float64, device="cuda").index_add(0, seq, u)
    pairs = -0.25 * torch.nn.functional.logsigmoid(BETA * (ratio[list(PAIRS[0])] - ratio[list(PAIRS[1])])).sum()
    rows = pk["src_row"][:N].long()
    q = torch.softmax(D(b["topk"][rows]) / T, 1)
    lp = torch.log_softmax(z / T, 1).gather(1, b["ids"][rows].long())
    kl = (q * (q.log() - lp)).sum(1)
    losses = [policy, pairs, (c * kl).sum() / N]
    parts = [torch.autograd.grad(v, y, retain_graph=True)[0] for v in losses]
    sum(losses).backward()
    return dict(losses=[v.detach() for v in losses], y=y.detach(), dy=sum(parts), norms=[v.norm() for v in parts], x=x.grad, head=p["head"].grad, wg=p["wg"].grad,
                wu=p["wu"].grad, wd=p["wd"].grad)


def test_objectives_on_packed_prefixes(batch):
    b = batch
    for seed in (0, 1):
        pk, N = _pack(b, seed)
        r, w = _run(b, pk, N), None
        w = _want(b, pk, N, r)
        rel = lambda a, t, size=None: float((a.double() - t).norm() / (t.norm() if size is None else size))   # noqa: E731
        assert rel(r["y"], w["y"]) <= 3 * STEP
        for o, v in zip(r["o"], w["losses"]):
            # y off by 3 STEP at most moves the loss by its gradient times that; the sums themselves are float64
            assert abs(float(o["loss"]) - float(v)) <= 3 * STEP * float(w["y"].norm() * sum(w["norms"])), float(v)
        size = float(sum(w["norms"]))
        # entries and results 2 STEP, the sum's rounding 1, and what y's 3 STEP do to the softmax (its slope is at most
        # as long as the gradient's own terms)
        assert rel(r["dy"], w["dy"], size) <= 6 * STEP
        amplified = size / float(w["dy"].norm())
        for got, want in ((r["g"]["dx"], w["x"]), (r["g"]["dw_gate"], w["wg"]), (r["g"]["dw_up"], w["wu"]),
                          (r["g"]["dw_down"], w["wd"])):
            assert rel(got, want) <= (6 * amplified + 4) * STEP
        parts = [objective.policy_loss, objective.preference_loss, objective.distill_loss]
        assert len(parts) == 3 and rel(r["dw"], w["head"]) <= 8 * max(1.0, amplified) * STEP


def test_accumulated_head_gradient_is_the_sum(batch):
    """The three calls adding to one buffer, against each alone."""
    b = batch
    pk, N = _pack(b, 2)
    r = _run(b, pk, N)
    rows = pk["src_row"][:N].long()
    chosen, rejected = (torch.tensor(p, dtype=torch.int32, device="cuda") for p in PAIRS)
    new = lambda: torch.empty_like(r["dw"])   # noqa: E731
    alone = [objective.policy_loss(r["y"], b["head"], pk["target"], r["old"], pk["weight"], pk["seq_id"], b["adv"], N, EPS,
                                   EPS, 1.0 / N, logp_ref=r["ref"], kl_coef=COEF, d_w_head=new()),
             objective.preference_loss(r["y"], b["head"], pk["target"], pk["cu_seqlens"], chosen, rejected, N, BETA, 0.25,
                                       logp_ref=r["ref"], d_w_head=new()),
             objective.distill_loss(r["y"], b["head"], b["ids"][rows].contiguous(), b["topk"][rows].contiguous(), N,
                                    1.0 / N, weight=pk["weight"], temperature=T, d_w_head=new())]
    want = sum(o["d_w_head"].double() for o in alone)
    size = sum(o["d_w_head"].double().abs() for o in alone)
    assert ((r["dw"].double() - want).abs() <= 3 * 2.0 ** -24 * size + 1e-30).all()
    for o, p in zip(r["o"], alone):
        assert torch.equal(o["loss"], p["loss"])


def test_the_penalty_left_out_is_the_clipped_loss(batch):
    """Without a penalty the policy loss is the clipped loss of the head call, whose gradients are float32."""
    b = batch
    pk, N = _pack(b, 3)
    r = _run(b, pk, N)
    args = (r["y"], b["head"], pk["target"], r["old"], pk["weight"], pk["seq_id"], b["adv"], N, EPS, EPS, 1.0 / N)
    a, want = objective.policy_loss(*args), pspo.loss_fwd_bwd(*args)
    # log-probs: the logits' sums in another order, (d + 2) 2^-24 of their terms, and the softmax's
    assert (a["logp_new"] - want["logp_new"]).abs().max() <= 2 * (b["cfg"].d + 66) * 2.0 ** -24 * 20
    assert abs(float(a["loss"] - want["loss"])) <= 1e-4 * float(want["stats"][0])
    assert int(a["stats"][2]) == int(want["stats"][1])
    for n in ("d_hidden", "d_w_head"):   # entries, scaled rows and results to bf16 here
        assert float((a[n].float() - want[n]).norm()) <= 3 * STEP * float(want[n].norm())
