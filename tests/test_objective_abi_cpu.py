"""The objectives' C ABI without a GPU: every symbol of pspo_objective.h is exported and bound, the workspace sizes,
and the refusals, which come before any device work."""
import os
import re

import pytest

from paper_2606_29758_amd import objective, pspo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, WORKSPACE, UNSUPPORTED = 1, 3, 4
A, BIG = 0x10000, 1 << 60          # an aligned address that no refused call touches; room enough
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pspo.LIB_PATH):
        pytest.fail("libpspo.so is not built (run __graft_entry__.build())")
    return objective.load()


def test_exports_every_declared_symbol(lib):
    with open(os.path.join(ROOT, "include", "pspo_objective.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pspo_[a-z_]+)\s*\(", text)))
    assert names == sorted(objective.exported_symbols()) and len(names) == 6
    for n in names:
        assert hasattr(lib, n), n


def test_flags_are_the_header_s():
    with open(os.path.join(ROOT, "include", "pspo_objective.h")) as f:
        text = f.read()
    value = lambda n: int(re.search(r"#define %s\s+(\d+)u?\b" % n, text).group(1))   # noqa: E731
    assert (value("PSPO_OBJ_DH_F32"), value("PSPO_OBJ_DW_F32"), value("PSPO_PREF_AVERAGE")) == (
        objective.DH_F32, objective.DW_F32, objective.PREF_AVERAGE)
    assert {k: value("PSPO_KL_" + k.upper()) for k in objective.KL_KINDS} == objective.KL_KINDS
    assert {k: value("PSPO_PREF_" + k.upper()) for k in objective.PREFERENCES} == objective.PREFERENCES


def _says(lib, rc, want, text):
    assert rc == want, (rc, lib.pspo_last_error())
    assert text in lib.pspo_last_error().decode(), lib.pspo_last_error()


ENDS = dict(loss=A, dh=A, dw=A)
POLICY = dict(h=A, w=A, target=A, old=A, ref=A, weight=A, seq=A, adv=A, N=4, d=64, V=100, R=2, lo=0.2, hi=0.2, coef=0.1, kl=3,
              T=1.0, scale=1.0, flags=0, **ENDS, logp=A, stats=A, err=None, ws=A, n=BIG)
PREF = dict(h=A, w=A, target=A, ref=A, weight=A, cu=A, chosen=A, rejected=A, N=4, d=64, V=100, R=2, P=1, kind=0, beta=0.1,
            smooth=0.1, T=1.0, scale=1.0, flags=0, **ENDS, logp=A, ratio=A, margin=A, err=None, ws=A, n=BIG)
DISTILL = dict(h=A, w=A, ids=A, t=A, weight=A, N=4, d=64, V=100, k=5, T=1.0, scale=1.0, flags=0, **ENDS, kl=A, err=None, ws=A,
               n=BIG)


def policy(lib, **kw):
    return lib.pspo_policy_loss_fwd_bwd(*dict(POLICY, **kw).values(), None)


def pref(lib, **kw):
    return lib.pspo_preference_fwd_bwd(*dict(PREF, **kw).values(), None)


def distill(lib, **kw):
    return lib.pspo_distill_fwd_bwd(*dict(DISTILL, **kw).values(), None)


SHARED = [
    (dict(N=-1), INVALID, "N must"), (dict(d=0), INVALID, "d and V"), (dict(V=0), INVALID, "d and V"),
    (dict(d=12), UNSUPPORTED, "multiple of 8"), (dict(d=(1 << 20) + 8), UNSUPPORTED, "at most"),
    (dict(V=(1 << 21) + 1), UNSUPPORTED, "at most"), (dict(N=(1 << 23) + 1, d=8, V=8), UNSUPPORTED, "at most"),
    (dict(N=1 << 23, d=8, V=(1 << 13) + 8), UNSUPPORTED, "at most"), (dict(N=1 << 23, d=(1 << 13) + 8, V=8), UNSUPPORTED, "at most"),
    (dict(V=1 << 21, d=1 << 16), UNSUPPORTED, "at most"),
    (dict(flags=1), INVALID, "float32 d_w_head"), (dict(flags=2), INVALID, "flag"), (dict(flags=1 << 20), INVALID, "flag"),
    (dict(T=0.0), INVALID, "temperature"), (dict(T=-1.0), INVALID, "temperature"), (dict(T=NAN), INVALID, "temperature"),
    (dict(T=INF), INVALID, "temperature"), (dict(T=1e-45), INVALID, "temperature"), (dict(scale=INF), INVALID, "loss_scale"),
    (dict(scale=NAN), INVALID, "loss_scale"), (dict(loss=None), INVALID, "loss"), (dict(loss=A + 4), INVALID, "loss"),
    (dict(dh=A + 8), INVALID, "16-byte"), (dict(dw=A + 2), INVALID, "16-byte"), (dict(err=A + 1), INVALID, "err_flag"),
    (dict(ws=A + 128), INVALID, "256-byte"), (dict(ws=None), INVALID, "workspace"), (dict(n=100), WORKSPACE, "too small"),
    (dict(h=None), INVALID, "null"), (dict(w=None), INVALID, "null"), (dict(h=A + 8), INVALID, "16-byte"),
    (dict(w=A + 2), INVALID, "16-byte"), (dict(weight=A + 2), INVALID, "misaligned")]


@pytest.mark.parametrize("kw,want,text", SHARED)
def test_refusals_of_all_three(lib, kw, want, text):
    for call in (policy, pref, distill):
        _says(lib, call(lib, **kw), want, text)


@pytest.mark.parametrize("kw,text", [
    (dict(R=0), "R must"), (dict(R=-1), "R must"), (dict(lo=1.0), "eps"), (dict(lo=-0.1), "eps"), (dict(hi=NAN), "eps"),
    (dict(hi=1.5), "eps"), (dict(coef=NAN), "kl_coef"), (dict(coef=INF), "kl_coef"), (dict(kl=0), "kl_kind"),
    (dict(kl=4), "kl_kind"), (dict(ref=None), "logp_ref"), (dict(target=None), "null"), (dict(old=None), "null"),
    (dict(weight=None), "null"), (dict(seq=None), "null"), (dict(adv=None), "null"), (dict(old=A + 1), "misaligned"),
    (dict(ref=A + 2), "misaligned"), (dict(stats=A + 4), "misaligned"), (dict(logp=A + 2), "misaligned"),
    (dict(flags=8192), "flag")])
def test_policy_refusals(lib, kw, text):
    _says(lib, policy(lib, **kw), INVALID, text)


@pytest.mark.parametrize("kw,text", [
    (dict(R=-1), "R and P"), (dict(P=-1), "R and P"), (dict(kind=2), "kind"), (dict(kind=-1), "kind"), (dict(beta=0.0), "beta"),
    (dict(beta=-1.0), "beta"), (dict(beta=NAN), "beta"), (dict(beta=1e-45), "beta"), (dict(smooth=-0.1), "smoothing"),
    (dict(smooth=1.1), "smoothing"), (dict(smooth=NAN), "smoothing"), (dict(kind=1), "smoothing belongs"),
    (dict(cu=None), "null"), (dict(chosen=None), "null"), (dict(rejected=None), "null"), (dict(target=None), "null"),
    (dict(cu=A + 2), "misaligned"), (dict(chosen=A + 1), "misaligned"), (dict(margin=A + 2), "misaligned"),
    (dict(ratio=A + 2), "misaligned")])
def test_preference_refusals(lib, kw, text):
    _says(lib, pref(lib, **kw), INVALID, text)


@pytest.mark.parametrize("R,P", [((1 << 23) + 1, 1), (1 << 23, (1 << 13) + 1), (1 << 20, 1 << 20)])
def test_preference_limits(lib, R, P):
    """What a launch cannot hold, or sequences that would look at more pairs than a call should."""
    assert objective.preference_workspace_bytes(4, 64, 100, R, P) == 0
    _says(lib, pref(lib, R=R, P=P), UNSUPPORTED, "R is at most")
    for r, p in ((1 << 23, 1 << 13), (1, 2 ** 31 - 1)):
        assert objective.preference_workspace_bytes(4, 64, 100, r, p) > 0
        _says(lib, pref(lib, R=r, P=p, n=100), WORKSPACE, "too small")


@pytest.mark.parametrize("kw,want,text", [
    (dict(k=0), UNSUPPORTED, "k must"), (dict(k=65), UNSUPPORTED, "k must"), (dict(k=-1), UNSUPPORTED, "k must"),
    (dict(ids=None), INVALID, "null"), (dict(t=None), INVALID, "null"), (dict(ids=A + 2), INVALID, "misaligned"),
    (dict(t=A + 1), INVALID, "misaligned"), (dict(kl=A + 2), INVALID, "misaligned"), (dict(flags=8192), INVALID, "flag")])
def test_distill_refusals(lib, kw, want, text):
    _says(lib, distill(lib, **kw), want, text)


def test_workspace_sizes(lib):
    """0 for what the calls refuse; never less for fewer rows; without gradients no more than with them."""
    p, q, k = objective.policy_loss_workspace_bytes, objective.preference_workspace_bytes, objective.distill_workspace_bytes
    for bad in (lambda: p(-1, 64, 100), lambda: p(4, 12, 100), lambda: p(4, 64, 0), lambda: p(1 << 23, 64, 1 << 21), lambda: p((1 << 23) + 1, 8, 8),
                lambda: q(4, 64, 100, -1, 1), lambda: q(4, 64, 100, 1, -1), lambda: k(4, 64, 100, 0), lambda: k(4, 64, 100, 65)):
        assert bad() == 0
    for d, V in ((64, 100), (1536, 151936), (520, 32003), (8, 1)):
        before = 0
        for N in (0, 1, 2, 16, 63, 64, 65, 66, 128, 200, 256, 257, 777, 1025, 4096, 4999, 8192, 20000):
            now = p(N, d, V)
            assert now >= before >= 0 and p(N, d, V, False) <= now
            assert q(N, d, V, 10, 20) >= now and k(N, d, V, 16) >= now
            before = now
    # 2 bytes an entry, and little beside it
    assert p(8192, 3584, 152064) < 1.3 * 2 * 8192 * 152064


@pytest.mark.parametrize("n", (2 ** 31, 2 ** 32 + 8))
def test_sizes_past_32_bits(n):
    for call in (lambda: objective.policy_loss_workspace_bytes(n, 8, 8), lambda: objective.distill_workspace_bytes(8, n, 8, 1),
                 lambda: objective.preference_workspace_bytes(8, 8, 8, 1, n)):
        with pytest.raises(ValueError, match="at most 2147483647"):
            call()
