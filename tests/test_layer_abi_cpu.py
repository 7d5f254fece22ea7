"""The layer operators' C ABI without a GPU: every symbol of pspo_layer.h is exported and bound, the
workspace sizes, and the refusals, which come before any device work."""
import ctypes
import os
import re

import pytest
import torch

from paper_2606_29758_amd import layer, pspo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, WORKSPACE, UNSUPPORTED, HIP = 0, 1, 3, 4, 5
A = 0x10000          # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pspo.LIB_PATH):
        pytest.fail("libpspo.so is not built (run __graft_entry__.build())")
    return layer.load()


def test_exports_every_declared_symbol(lib):
    with open(os.path.join(ROOT, "include", "pspo_layer.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pspo_[a-z_]+)\s*\(", text)))
    assert names == sorted(layer.exported_symbols()) and len(names) == 8
    for n in names:
        assert hasattr(lib, n), n


def _says(lib, rc, want, text):
    assert rc == want, (rc, lib.pspo_last_error())
    assert text in lib.pspo_last_error().decode(), lib.pspo_last_error()


QK = dict(q=A, k=A, qs=256, ks=128, qw=A, kw=A, inv=A, pos=A, seq=None, cu=None, first=None, N=4, R=0, Hq=2, Hk=1, D=128,
          rot=128, eps=1e-6, type=0, flags=0)
QK_ORDER = ("q", "k", "qs", "ks", "qw", "kw", "inv", "pos", "seq", "cu", "first", "N", "R", "Hq", "Hk", "D", "rot", "eps",
            "type", "flags")


def _qk_fwd(lib, qo=A, ko=A, err=None, **kw):
    v = dict(QK, **kw)
    return lib.pspo_qk_norm_rope_fwd(*[v[k] for k in QK_ORDER], qo, ko, err, None)


def _qk_bwd(lib, dqo=A, dko=A, dq=A, dk=A, dqw=A, dkw=A, ws=A, n=1 << 30, **kw):
    v = dict(QK, **kw)
    return lib.pspo_qk_norm_rope_bwd(dqo, dko, *[v[k] for k in QK_ORDER], dq, dk, dqw, dkw, None, ws, n, None)


@pytest.mark.parametrize("kw,want,text", [
    (dict(N=-1), INVALID, "N and R"), (dict(R=-2), INVALID, "N and R"), (dict(Hq=0), INVALID, "heads_q"),
    (dict(Hk=-1), INVALID, "heads"), (dict(Hq=70000, qs=1 << 30), UNSUPPORTED, "65536"),
    (dict(D=0), UNSUPPORTED, "head_dim"), (dict(D=12), UNSUPPORTED, "head_dim"),
    (dict(D=520, qs=2048, ks=2048), UNSUPPORTED, "head_dim"), (dict(rot=-16), UNSUPPORTED, "rot_dim"),
    (dict(rot=24), UNSUPPORTED, "rot_dim"), (dict(rot=144), UNSUPPORTED, "rot_dim"), (dict(flags=4), INVALID, "flag"),
    (dict(type=2), INVALID, "element type"), (dict(eps=0.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"), (dict(flags=2), INVALID, "weights need"), (dict(qs=255), INVALID, "strides"),
    (dict(ks=120), INVALID, "strides"), (dict(qs=260), INVALID, "16-byte"), (dict(qs=1 << 41), INVALID, "range"),
    (dict(N=1 << 27), UNSUPPORTED, "tokens"), (dict(q=None), INVALID, "null input"), (dict(k=None), INVALID, "null input"),
    (dict(q=A + 2), INVALID, "misaligned"), (dict(kw=A + 4), INVALID, "misaligned"), (dict(inv=None), INVALID, "inv_freq"),
    (dict(pos=None), INVALID, "positions"), (dict(pos=None, seq=A), INVALID, "positions")])
def test_qk_refusals(lib, kw, want, text):
    _says(lib, _qk_fwd(lib, **kw), want, text)
    _says(lib, _qk_bwd(lib, **kw), want, text)


def test_qk_refusals_of_outputs(lib):
    _says(lib, _qk_fwd(lib, qo=None), INVALID, "null output")
    _says(lib, _qk_fwd(lib, ko=None), INVALID, "null output")
    _says(lib, _qk_fwd(lib, qo=A + 8), INVALID, "misaligned")
    _says(lib, _qk_bwd(lib, dqo=None), INVALID, "null pointer")
    _says(lib, _qk_bwd(lib, dk=None), INVALID, "null pointer")
    _says(lib, _qk_bwd(lib, qw=None), INVALID, "weight's gradient")
    _says(lib, _qk_bwd(lib, dqw=A + 2), INVALID, "misaligned")
    _says(lib, _qk_bwd(lib, ws=None), INVALID, "workspace")
    _says(lib, _qk_bwd(lib, n=8), WORKSPACE, "smaller")
    assert _qk_fwd(lib, N=0, q=None, k=None, qo=None, ko=None) == OK
    assert lib.pspo_qk_norm_rope_workspace_bytes(4, 128) == 1 * 2 * 128 * 4
    assert lib.pspo_qk_norm_rope_workspace_bytes(10 ** 6, 128) == 1024 * 2 * 128 * 4
    assert lib.pspo_qk_norm_rope_workspace_bytes(-1, 128) == 0


def test_dropout_refusals(lib):
    f = lambda x=A, res=A, rows=A, N=4, d=64, p=0.1, ty=0, y=A: lib.pspo_dropout_add_fwd(   # noqa: E731
        x, res, rows, N, d, p, 1, 2, ty, y, None)
    b = lambda ti=0, to=1, dy=A, dx=A: lib.pspo_dropout_bwd(dy, A, 4, 64, 0.1, 1, 2, ti, to, dx, None)   # noqa: E731
    _says(lib, f(N=-1), INVALID, "N must")
    _says(lib, f(d=0), UNSUPPORTED, "d % 8")
    _says(lib, f(d=12), UNSUPPORTED, "d % 8")
    for p in (-0.1, 1.0, float("nan"), float("inf")):
        _says(lib, f(p=p), INVALID, "p must")
    _says(lib, f(ty=7), INVALID, "element type")
    _says(lib, f(x=None), INVALID, "null")
    _says(lib, f(y=None), INVALID, "null")
    _says(lib, f(res=A + 8), INVALID, "misaligned")
    _says(lib, f(rows=A + 1), INVALID, "misaligned")
    _says(lib, b(ti=3), INVALID, "element type")
    _says(lib, b(to=-1), INVALID, "element type")
    _says(lib, b(dx=A + 2), INVALID, "misaligned")
    assert f(N=0, x=None, y=None) == OK


def test_gated_ffn_refusals(lib):
    big = 1 << 40
    f = lambda x=A, wg=A, N=100, d=64, fd=72, act=0, y=A, pre=None, ws=A, n=big: lib.pspo_gated_ffn_fwd(   # noqa: E731
        x, wg, A, A, N, d, fd, act, y, pre, ws, n, None)
    b = lambda dy=A, pre=None, N=100, d=64, fd=72, act=0, fl=0, dx=A, dw=A, ws=A, n=big: lib.pspo_gated_ffn_bwd(   # noqa: E731
        dy, A, A, A, A, pre, N, d, fd, act, fl, dx, dw, A, A, ws, n, None)
    for g in (f, b):
        _says(lib, g(N=-1), INVALID, "N must")
        _says(lib, g(d=60), UNSUPPORTED, "d % 8")
        _says(lib, g(fd=0), UNSUPPORTED, "f > 0")
        _says(lib, g(fd=(1 << 20) + 8), UNSUPPORTED, "2^20")
        _says(lib, g(act=2), INVALID, "activation")
        _says(lib, g(ws=None), INVALID, "null")
        _says(lib, g(ws=A + 16), INVALID, "misaligned")
        _says(lib, g(pre=A + 4), INVALID, "misaligned")
        _says(lib, g(n=64), WORKSPACE, "smaller")
    _says(lib, f(x=None), INVALID, "null")
    _says(lib, f(wg=A + 2), INVALID, "misaligned")
    _says(lib, b(dx=None), INVALID, "null")
    _says(lib, b(dw=None), INVALID, "null")
    _says(lib, b(fl=2), INVALID, "flag")
    _says(lib, b(fl=1), INVALID, "float32")
    assert f(N=0, x=None, y=None, ws=None) == OK


@pytest.mark.parametrize("N,d,f", [(0, 64, 72), (1, 64, 72), (64, 1536, 6144), (777, 1000, 4104), (8192, 3584, 14336),
                                   (2 ** 31 - 1, 2 ** 20, 2 ** 20)])
def test_gated_ffn_workspace(lib, N, d, f):
    """The forward holds the intermediate, the backward its gradients too; more only for the slabs (at most
    256 MB a product) and the pre-activations where they are computed again."""
    size = lambda **kw: layer.gated_ffn_workspace_bytes(N, d, f, **kw)   # noqa: E731
    fwd, kept, own = size(), size(backward=True, preact=True), size(backward=True)
    slabs = (256 << 20) + 1024
    assert 2 * N * f <= fwd <= 2 * N * f + slabs
    assert 6 * N * f <= kept <= 6 * N * f + slabs
    assert 14 * N * f <= own <= 14 * N * f + slabs


def test_gated_ffn_workspace_of_refused_sizes(lib):
    for N, d, f in ((-1, 64, 64), (1, 0, 64), (1, 64, -8), (1, 1 << 21, 64)):
        assert layer.gated_ffn_workspace_bytes(N, d, f) == 0


def test_binding_refuses_host_tensors():
    x = torch.ones(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="torch.Tensor"):
        layer._type([1.0], "x")
    with pytest.raises(ValueError, match="must be \\[>= 5, 64\\]"):
        layer._rows(x, 5, (64,), "x")
    with pytest.raises(ValueError, match="device tensor"):
        layer._here(x, torch.bfloat16, "x", 0)
    with pytest.raises(ValueError, match="overlaps"):
        layer._apart(x, "out", None, x[1:2])
    layer._apart(x[:1], "out", x[1:])
    with pytest.raises(ValueError, match="N must"):
        layer._count(-1)
    assert isinstance(ctypes.c_void_p(layer._ptr(x)).value, int) and layer._ptr(None) is None
