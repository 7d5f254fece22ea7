"""The objectives' binding without a GPU: what it refuses by itself."""
import pytest
import torch

from paper_2606_29758_amd import layer, objective
from test_layer_binding_cpu import BF, F4, I4, Here, Shaped, _in, _new   # noqa: F401

N, d, V, R, P, K = 6, 16, 24, 3, 2, 4


@pytest.fixture
def device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def stop(*args, **kw):
        raise AssertionError("the call went past its checks")
    monkeypatch.setattr(objective, "_stream", stop)


SHAPES = dict(hidden=(BF, N, d), w_head=(BF, V, d), target=(I4, N), logp_old=(F4, N), weight=(F4, N), seq_id=(I4, N),
              advantage=(F4, R), logp_ref=(F4, N), cu_seqlens=(I4, R + 1), chosen=(I4, P), rejected=(I4, P), topk_ids=(I4, N, K),
              topk_logit=(F4, N, K), err_flag=(I4, 1))
CALLS = dict(
    policy=(["hidden", "w_head", "target", "logp_old", "weight", "seq_id", "advantage"], ["logp_ref", "err_flag"],
            lambda a, kw: objective.policy_loss(*a, kw.pop("N", N), 0.2, 0.2, 1.0, kl_coef=0.1, **kw)),
    pref=(["hidden", "w_head", "target", "cu_seqlens", "chosen", "rejected"], ["logp_ref", "weight", "err_flag"],
          lambda a, kw: objective.preference_loss(*a, kw.pop("N", N), 0.1, 1.0, **kw)),
    distill=(["hidden", "w_head", "topk_ids", "topk_logit"], ["weight", "err_flag"],
             lambda a, kw: objective.distill_loss(*a, kw.pop("N", N), 1.0, **kw)))


def _call(which, change=None, **more):
    first, named, call = CALLS[which]
    change = change or {}
    a = [change[n] if n in change else _new(*SHAPES[n]) for n in first]
    return call(a, dict({n: change[n] if n in change else _new(*SHAPES[n]) for n in named}, **more))


def _arguments(which):
    return CALLS[which][0] + CALLS[which][1]


@pytest.mark.parametrize("which", CALLS)
def test_all_is_well_up_to_the_stream(which, device):
    with pytest.raises(AssertionError, match="past its checks"):
        _call(which)


@pytest.mark.parametrize("which,name", [(w, n) for w in CALLS for n in _arguments(w)])
def test_wrong_arguments_are_refused(which, name, device):
    dtype, *shape = SHAPES[name]
    wrong = torch.float64 if dtype != I4 else torch.int64
    with pytest.raises((TypeError, ValueError)):
        _call(which, {name: _new(wrong, *shape)})
    with pytest.raises((TypeError, ValueError)):
        _call(which, {name: torch.zeros(shape, dtype=dtype)})          # on the host
    with pytest.raises((TypeError, ValueError)):
        _call(which, {name: [1.0]})
    if name not in ("cu_seqlens", "advantage"):
        short = (0,) if name == "err_flag" else (shape[0] - 1, *shape[1:])
        if name not in ("w_head",):
            with pytest.raises(ValueError):
                _call(which, {name: _new(dtype, *short)})
        if shape[0] > 1:
            strided = torch.zeros((2 * shape[0], *shape[1:]), dtype=dtype)[::2].as_subclass(Here)
            with pytest.raises(ValueError):
                _call(which, {name: strided})
    else:
        with pytest.raises(ValueError):
            _call(which, {name: _new(dtype, *shape, 1)})


@pytest.mark.parametrize("which", CALLS)
def test_widths_have_to_agree(which, device):
    with pytest.raises(ValueError):
        _call(which, dict(hidden=_new(BF, N, d + 8)))
    with pytest.raises(ValueError):
        _call(which, N=N + 1)
    with pytest.raises(ValueError):
        _call(which, N=-1)
    with pytest.raises(ValueError, match="at most 2147483647"):
        _call(which, N=2 ** 32 + 1)
    with pytest.raises(ValueError, match="at most 2147483647"):
        _call(which, dict(w_head=Shaped.of((2 ** 32 + 8, d))))
    with pytest.raises(ValueError, match="d_w_head must be"):
        _call(which, d_w_head=_new(BF, V, d + 8))
    with pytest.raises(ValueError, match="d_hidden must be"):
        _call(which, d_hidden=_new(BF, N - 1, d))
    with pytest.raises(TypeError):
        _call(which, d_w_head=_new(torch.float16, V, d))
    with pytest.raises(TypeError):
        _call(which, d_hidden=_new(torch.float64, N, d))


@pytest.mark.parametrize("which", CALLS)
def test_what_is_given_has_to_be_wanted(which, device):
    with pytest.raises(ValueError, match="not wanted"):
        _call(which, d_w_head=_new(BF, V, d), want_head=False)
    with pytest.raises(ValueError, match="not wanted"):
        _call(which, d_hidden=_new(BF, N, d), want_hidden=False)
    with pytest.raises(ValueError, match="accumulate"):
        _call(which, accumulate=True)


def test_names_of_kinds(device):
    with pytest.raises(ValueError, match="kl must be one of"):
        _call("policy", kl="k4")
    with pytest.raises(ValueError, match="kind must be one of"):
        _call("pref", kind="hinge")


def test_pairs_of_one_length(device):
    with pytest.raises(ValueError, match="one length"):
        _call("pref", dict(chosen=_new(I4, P + 1)))


@pytest.mark.parametrize("which,name", [(w, n) for w in CALLS for n in _arguments(w)])
def test_outputs_and_workspace_stand_apart(which, name, device):
    m = torch.zeros(1 << 20, dtype=torch.uint8)
    dtype, *shape = SHAPES[name]
    change = {name: _in(m, dtype, *shape, at=64)}
    for kw in (dict(d_hidden=_in(m, F4, N, d)), dict(d_w_head=_in(m, F4, V, d)), dict(workspace=m.as_subclass(Here))):
        with pytest.raises(ValueError, match="overlaps"):
            _call(which, change, **kw)


@pytest.mark.parametrize("which", CALLS)
def test_outputs_stand_apart_from_each_other(which, device):
    m = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="overlaps"):
        _call(which, d_hidden=_in(m, F4, N, d), d_w_head=_in(m, BF, V, d, at=64))
    for kw in (dict(d_hidden=_in(m, F4, N, d)), dict(d_w_head=_in(m, BF, V, d))):
        with pytest.raises(ValueError, match="overlaps"):
            _call(which, workspace=m.as_subclass(Here), **kw)


def test_the_binding_shares_the_layer_s_checks():
    assert objective._here is layer._here and objective._apart is layer._apart
