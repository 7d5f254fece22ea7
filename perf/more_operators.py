"""Timed cases of the training objectives that go through the LM head beside the clipped loss: what a
program calls on the final hidden rows of a batch to get its loss and the gradients of the rows and the head.

Operators
  policy   the clipped policy loss with a penalty on the divergence from a reference policy
  pref     a preference loss on pairs of sequences (log ratios to a reference, summed or averaged)
  distill  distillation from a teacher's top logits

Widths, vocabularies and token counts are those of the repository's own workloads (d = 128, 1536 and 3584,
V = 2048, 151936 and 152064) or generic ones.  The softmax of the inputs ranges from flat to peaked, as a
trained policy's does.
"""
import math

import torch

own = False

DEV = "cuda"
COST = 2.7e13   # 6 N d V of the largest listed case


def listed():
    return [
        # one token of one completion: bound by the head's bytes
        dict(name="policy_token", op="policy", N=1, R=1, d=1536, V=151936, kl="k3", coef=0.05, T=1.0, masked=0.0,
             head=True),
        # a micro-batch of the 1.5B-shaped policy
        dict(name="policy_micro", op="policy", N=777, R=8, d=1536, V=151936, kl="k3", coef=0.05, T=1.0, masked=0.0,
             head=True),
        # odd everywhere, sampled at a temperature, a third of the rows masked
        dict(name="policy_odd", op="policy", N=1301, R=11, d=1000, V=50257, kl="k2", coef=0.1, T=0.7, masked=0.33,
             head=True),
        # a training batch of the 7B-shaped policy: the largest
        dict(name="policy_batch", op="policy", N=4999, R=64, d=3584, V=152064, kl="k1", coef=0.02, T=1.0, masked=0.0,
             head=True),
        # a few short pairs on the tiny workload's head: latency
        dict(name="pref_tiny", op="pref", N=257, R=8, P=4, d=128, V=2048, kind="sigmoid", beta=0.1, smooth=0.0,
             average=False, T=1.0, masked=0.2, head=True),
        # all pairs of eight completions of a prompt, length-normalised
        dict(name="pref_ranked", op="pref", N=1999, R=8, P=28, d=1536, V=151936, kind="squared", beta=0.5, smooth=0.0,
             average=True, T=1.0, masked=0.1, head=True),
        # thirty-two pairs, the head frozen (adapters are trained below it)
        dict(name="pref_batch", op="pref", N=8192, R=64, P=32, d=3584, V=152064, kind="sigmoid", beta=0.1, smooth=0.1,
             average=False, T=1.0, masked=0.0, head=False),
        # 16 tokens, the lists of 16 that a rollout engine reports
        dict(name="distill_few", op="distill", N=16, k=16, d=3584, V=152064, T=1.0, masked=0.0, head=True),
        # a micro-batch of a small student, softened
        dict(name="distill_soft", op="distill", N=1023, k=16, d=1536, V=151936, T=2.0, masked=0.1, head=True),
        # long lists with holes on an odd vocabulary
        dict(name="distill_odd", op="distill", N=2501, k=50, d=520, V=32003, T=1.0, masked=0.25, head=True),
        # a training batch
        dict(name="distill_batch", op="distill", N=4096, k=16, d=3584, V=152064, T=1.0, masked=0.0, head=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "pref", "distill"])
    d, V = 8 * _log_int(rng, 16, 512), _log_int(rng, 1000, 152064)
    N = max(1, min(_log_int(rng, 1, 16384), int(COST / (6.0 * d * V))))
    c = dict(op=op, N=N, d=d, V=V, T=rng.choice([1.0, 1.0, 0.7, 2.0]), masked=rng.choice([0.0, 0.0, 0.1, 0.4]),
             head=rng.random() < 0.8)
    if op == "policy":
        return dict(c, R=min(N, rng.choice([1, 5, 64])), kl=rng.choice(["k1", "k2", "k3"]),
                    coef=rng.choice([0.0, 0.02, 0.1]))
    if op == "pref":
        R = min(max(2, N // 8), rng.choice([2, 7, 64]))
        kind = rng.choice(["sigmoid", "sigmoid", "squared"])
        return dict(c, R=R, P=rng.choice([R // 2, R, 2 * R + 1]), kind=kind, average=kind == "squared",
                    beta=rng.choice([0.05, 0.1, 0.3]), smooth=rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0)
    return dict(c, k=rng.choice([1, 2, 5, 16, 16, 33, 64]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _log_probs(h, w, target, inv_t):
    """log softmax(h w^T inv_t) at the targets, float32."""
    wf = w.float()
    out = []
    for a in range(0, h.shape[0], 4096):
        z = h[a:a + 4096].float() @ wf.T * inv_t
        out.append(z.gather(1, target[a:a + 4096, None].long())[:, 0] - torch.logsumexp(z, 1))
    return torch.cat(out)


def _cuts(g, N, R):
    """Offsets of R sequences, none empty where there are tokens enough."""
    if R > N:
        return torch.sort(torch.randint(0, N + 1, (R + 1,), device=DEV, generator=g)).values
    inner = torch.randperm(N - 1, device=DEV, generator=g)[:R - 1] + 1 if R > 1 else torch.empty(0, device=DEV).long()
    ends = torch.tensor([0, N], device=DEV)
    return torch.sort(torch.cat([ends, inner])).values


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    rand = lambda *n: torch.rand(*n, device=DEV, generator=g)      # noqa: E731
    randn = lambda *n: torch.randn(*n, device=DEV, generator=g)    # noqa: E731
    N, d, V = case["N"], case["d"], case["V"]
    w = (randn(V, d) * (1.2 / math.sqrt(d))).to(torch.bfloat16)
    target = torch.randint(0, V, (N,), device=DEV, generator=g).to(torch.int32)
    # the target's logit ranges from the others' (a flat softmax) to 6 above what all of them weigh together (a
    # peaked one; not for a few tokens alone, whose log-probs near 0 have no digits left in 32 bits)
    up = w[target.long()].float()
    top = math.log(V) + (6 if N > 32 else 1)
    h = randn(N, d) + up * (top * rand(N) / up.square().sum(1).clamp_min(1e-6))[:, None]
    s = dict(case=dict(case), w=w, h=h.to(torch.bfloat16), target=target,
             weight=1 + 7 * rand(N) ** 4)   # 1 / (probability that a prefix reaches the token)
    off = rand(N) < case["masked"]
    if case["op"] == "pref":
        s["weight"] = torch.ones(N, device=DEV)
    s["weight"][off] = 0.0
    if case["op"] != "distill":
        l = _log_probs(s["h"], w, target, 1 / case["T"])
        cu = _cuts(g, N, case["R"])
        s["cu"] = cu.to(torch.int32)
        # the trained policy has moved from its reference: up where it was rewarded
        seq = torch.bucketize(torch.arange(N, device=DEV), cu[1:], right=True).clamp_max(case["R"] - 1)
        s["seq"] = seq.to(torch.int32)
        s["ref"] = l - (0.08 * randn(case["R"]))[seq] - 0.2 * randn(N)
        s["ref"][off] = float("-inf")
    if case["op"] == "policy":
        r = 0.1 * randn(N)
        for edge in (math.log(0.8), math.log(1.2)):   # a ratio on the clip's border is no test of anything
            near = (r - edge).abs() < 1e-3
            r = torch.where(near, edge + torch.where(r < edge, -2e-3, 2e-3), r)
        s["old"] = l - r
        s["old"][off] = float("nan")
        s["adv"] = randn(case["R"]) + 0.5   # the batch did better than its baseline: the loss is no cancelled sum
    if case["op"] == "pref":
        R, P = case["R"], case["P"]
        a = torch.randint(0, R, (P,), device=DEV, generator=g)
        b = (a + 1 + torch.randint(0, R - 1, (P,), device=DEV, generator=g)) % R
        s["chosen"], s["rejected"] = a.to(torch.int32), b.to(torch.int32)
    if case["op"] == "distill":
        k = case["k"]
        # distinct ids: an arithmetic run modulo the vocabulary, the target first
        step = 1 + torch.randint(0, max(1, (V - 1) // k), (N, 1), device=DEV, generator=g)
        s["ids"] = ((target[:, None].long() + step * torch.arange(k, device=DEV)) % V).to(torch.int32)
        t = torch.sort(4 * randn(N, k), dim=1, descending=True).values + 3 * rand(N, 1)
        s["teacher"] = t
        if case["masked"]:   # lists of different lengths
            hole = torch.arange(k, device=DEV) >= 1 + (k * rand(N, 1)).int()
            s["ids"][hole] = -1
            s["teacher"][hole] = float("nan")
    s["h"][off] = float("nan")
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _own(s):
    from paper_2606_29758_amd import objective
    c = s["case"]
    N = c["N"]
    kw = dict(temperature=c["T"], want_head=c["head"])
    if c["op"] == "policy":
        o = objective.policy_loss(s["h"], s["w"], s["target"], s["old"], s["weight"], s["seq"], s["adv"], N, 0.2, 0.2,
                                  1.0 / N, logp_ref=s["ref"], kl_coef=c["coef"], kl=c["kl"], **kw)
        more = [o["logp_new"]]
    elif c["op"] == "pref":
        cu = s["cu"]
        if c["R"] > N:   # offsets that may leave the rows out: those of the sequences that they are counted in
            cu = torch.searchsorted(s["seq"], torch.arange(c["R"] + 1, dtype=torch.int32, device=DEV), out_int32=True)
        o = objective.preference_loss(s["h"], s["w"], s["target"], cu, s["chosen"], s["rejected"], N, c["beta"],
                                      1.0 / c["P"], logp_ref=s["ref"], weight=s["weight"], kind=c["kind"],
                                      smoothing=c["smooth"], average=c["average"], **kw)
        more = [o["logp_new"], o["seq_ratio"]]
    else:
        o = objective.distill_loss(s["h"], s["w"], s["ids"], s["teacher"], N, 1.0 / N, weight=s["weight"], **kw)
        more = [o["kl"]]
    return [o["loss"].float(), *more, o["d_hidden"]] + ([o["d_w_head"]] if c["head"] else [])


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------

def _policy_terms(s, c, l, on):
    """Loss and its derivative to each token's log-prob."""
    weight = s["weight"].double() / c["N"]
    A = s["adv"].double()[s["seq"].long()]
    zero = torch.zeros_like(l)
    rho = torch.exp(torch.where(on, l - s["old"], zero))
    clipped = rho.clamp(0.8, 1.2)
    inside = torch.where(A > 0, rho <= 1.2, rho >= 0.8) & (A != 0)
    u = torch.where(on, l - s["ref"], zero)   # log p - log ref
    if c["kl"] == "k1":
        kl, dkl = u, torch.ones_like(u)
    elif c["kl"] == "k2":
        kl, dkl = 0.5 * u * u, u
    else:
        kl, dkl = torch.expm1(-u) + u, -torch.expm1(-u)
    loss = (weight * (c["coef"] * kl - torch.minimum(rho * A, clipped * A))).sum()
    return loss, weight * (c["coef"] * dkl - torch.where(inside, rho * A, zero))


def _pref_terms(s, c, l, on):
    R = c["R"]
    seq = s["seq"].long()
    weight = s["weight"].double()
    ratio = torch.where(on, (l - s["ref"]) * weight, torch.zeros_like(l))
    sums = torch.zeros(R, dtype=torch.float64, device=l.device).index_add_(0, seq, ratio)
    norm = torch.ones(R, dtype=torch.float64, device=l.device)
    if c["average"]:
        total = torch.zeros_like(norm).index_add_(0, seq, weight)
        norm = torch.where(total > 0, 1 / total.clamp_min(1e-30), torch.zeros_like(total))
    sums = sums * norm
    a, b = s["chosen"].long(), s["rejected"].long()
    u = sums[a] - sums[b]
    beta, eps = c["beta"], c["smooth"]
    if c["kind"] == "sigmoid":
        x = beta * u
        soft = lambda y: torch.log1p(torch.exp(-y.abs())) + (-y).clamp_min(0)   # -log sigmoid(y)   # noqa: E731
        loss = ((1 - eps) * soft(x) + eps * soft(-x)).sum() / c["P"]
        du = beta * (eps * torch.sigmoid(x) - (1 - eps) * torch.sigmoid(-x)) / c["P"]
    else:
        loss = (u - 0.5 / beta).square().sum() / c["P"]
        du = 2 * (u - 0.5 / beta) / c["P"]
    coef = torch.zeros_like(norm).index_add_(0, a, du).index_add_(0, b, -du) * norm
    return loss, coef[seq] * weight, sums.float()


def _plain(s):
    c = s["case"]
    N, inv_t = c["N"], 1 / c["T"]
    on = s["weight"] != 0
    if c["op"] == "distill":
        valid = s["ids"] >= 0
        on = on & valid.any(1)
        ids = torch.where(valid, s["ids"], torch.zeros_like(s["ids"])).long()
    else:
        ids = s["target"].long()[:, None]
    h = torch.where(on[:, None], s["h"].float(), torch.zeros((), device=DEV))
    w = s["w"].float()
    z = (h @ w.T).mul_(inv_t)
    if c["op"] == "distill":
        zt = z.gather(1, ids)
    else:   # in 64 bits: long sums of log-probs follow
        zt = (h.double() * w[ids[:, 0]].double()).sum(1, keepdim=True) * inv_t
    m = z.amax(1, keepdim=True)
    p = torch.exp_(z.sub_(m))
    total = p.sum(1, keepdim=True, dtype=torch.float64)
    lse = m.double() + torch.log(total)
    p.div_(total)
    # p becomes the logit gradient
    if c["op"] == "distill":
        t = torch.where(valid, s["teacher"] * inv_t, torch.full_like(s["teacher"], float("-inf")))
        t = torch.where(on[:, None], t, torch.zeros_like(t))
        tm = t.amax(1, keepdim=True)
        q = torch.exp(t - tm)
        q = q / q.sum(1, keepdim=True)
        log_q = torch.log(torch.where(q > 0, q, torch.ones_like(q)))
        kl = torch.where(valid & (q > 0), q * (log_q - zt + lse.float()), torch.zeros_like(q)).sum(1)
        kl = torch.where(on, kl, torch.zeros_like(kl))
        scale = torch.where(on, s["weight"] / N, torch.zeros_like(kl))
        loss = (scale.double() * kl.double()).sum()
        more = [kl]
        p.scatter_add_(1, ids, torch.where(valid, -q, torch.zeros_like(q)))
        p.mul_((scale * inv_t)[:, None])
    else:
        l = (zt - lse)[:, 0]   # in 64 bits from here on
        if c["op"] == "policy":
            loss, delta = _policy_terms(s, c, l, on)
            more = []
        else:
            loss, delta, sums = _pref_terms(s, c, l, on)
            more = [sums]
        more = [torch.where(on, l, torch.zeros_like(l)).float(), *more]
        # (p - 1 from the log-prob: no cancellation where p is near 1)
        p.scatter_(1, ids, torch.expm1(l).float()[:, None])
        p.mul_((-delta * inv_t).float()[:, None])
    dh = (p @ w).to(torch.bfloat16)
    out = [loss.float().reshape(1), *more, dh]
    if c["head"]:
        out.append((p.T @ h).to(torch.bfloat16))
    return out


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    N, d, V = case["N"], case["d"], case["V"]
    moved = 2.0 * V * d + 4.0 * N * d + (2.0 * V * d if case["head"] else 0.0)
    moved += 8.0 * N * case["k"] if case["op"] == "distill" else 24.0 * N
    return {"bytes": moved, "flops": (6.0 if case["head"] else 4.0) * N * d * V}


# ---------------------------------------------------------------------------
# the definition in 64 bits, differentiated block by block
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    N, R, T = case["N"], case.get("R"), case["T"]
    w = s["w"].double().requires_grad_(case["head"])
    rows = torch.nonzero(s["weight"] != 0)[:, 0]
    if case["op"] == "distill":
        rows = rows[(s["ids"][rows] >= 0).any(1)]
    h = s["h"][rows].double()
    step = 1024

    def quantity(hb, at):
        """What the loss takes from each row: its log-prob, or its divergence from the teacher."""
        lp = torch.log_softmax(hb @ w.T / T, 1)
        if case["op"] != "distill":
            return lp.gather(1, s["target"][at, None].long())[:, 0]
        ids, there = s["ids"][at].long(), s["ids"][at] >= 0
        lq = torch.log_softmax(s["teacher"][at].double().masked_fill(~there, -float("inf")) / T, 1)
        lq = lq.masked_fill(~there, 0)
        each = lq.exp() * (lq - lp.gather(1, ids.clamp_min(0)))
        return each.masked_fill(~there, 0).sum(1)

    with torch.no_grad():
        x = torch.cat([quantity(h[a:a + step], rows[a:a + step]) for a in range(0, len(rows), step)] +
                      [torch.empty(0, dtype=torch.float64, device=DEV)])
    x.requires_grad_(True)
    c = s["weight"][rows].double()
    more = []
    if case["op"] == "distill":
        loss = (c * x).sum() / N
    elif case["op"] == "policy":
        A = s["adv"].double()[s["seq"][rows].long()]
        rho = torch.exp(x - s["old"][rows].double())
        gain = torch.minimum(rho * A, rho.clamp(0.8, 1.2) * A)
        u = x - s["ref"][rows].double()
        kl = u if case["kl"] == "k1" else u ** 2 / 2 if case["kl"] == "k2" else torch.exp(-u) - 1 + u
        loss = (c * (case["coef"] * kl - gain)).sum() / N
    else:
        seq = torch.nn.functional.one_hot(s["seq"][rows].long(), R).double() * c[:, None]
        if case["average"]:
            seq = seq / seq.sum(0).masked_fill(seq.sum(0) == 0, 1)
        ratio = (x - s["ref"][rows].double()) @ seq
        u = ratio[s["chosen"].long()] - ratio[s["rejected"].long()]
        if case["kind"] == "sigmoid":
            ls, e = torch.nn.functional.logsigmoid, case["smooth"]
            loss = -((1 - e) * ls(case["beta"] * u) + e * ls(-case["beta"] * u)).mean()
        else:
            loss = ((u - 1 / (2 * case["beta"])) ** 2).mean()
        more = [ratio.detach()]
    loss.backward()
    dh = torch.zeros((N, case["d"]), dtype=torch.float64, device=DEV)
    for a in range(0, len(rows), step):
        hb = h[a:a + step].detach().requires_grad_(True)
        (quantity(hb, rows[a:a + step]) * x.grad[a:a + step]).sum().backward()
        dh[rows[a:a + step]] = hb.grad
    each = torch.zeros(N, dtype=torch.float64, device=DEV)
    each[rows] = x.detach()
    out = [loss.detach().reshape(1), each, *more, dh]
    if case["head"]:
        out.append(w.grad if w.grad is not None else torch.zeros_like(w))
    return out
