"""The layer binding's own checks, without a GPU."""
import pytest
import torch

from paper_2606_29758_amd import layer

BIG = (2 ** 31, 2 ** 32 + 5)   # the C calls take 32-bit counts, and ctypes would pass the low bits alone


class Shaped(torch.Tensor):
    """A tensor that reports a shape no host could hold, on the current device."""

    @staticmethod
    def of(shape, dtype=torch.bfloat16):
        t = torch.empty(1, dtype=dtype).as_subclass(Shaped)
        t.faked = torch.Size(shape)
        return t

    shape = property(lambda self: self.faked)
    is_cuda = property(lambda self: True)

    def dim(self):
        return len(self.faked)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def stride(self, i=None):
        s = [1]
        for n in self.faked[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]


@pytest.fixture
def device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def stop(*args, **kw):
        raise AssertionError("the call went past its checks")
    monkeypatch.setattr(layer, "_stream", stop)


@pytest.mark.parametrize("n", BIG)
def test_counts_past_32_bits_are_refused(n, device):
    x, w = Shaped.of((n, 64)), Shaped.of((72, 64))
    q = Shaped.of((n, 2, 64))
    for call in (lambda: layer.dropout_add(x, n, 0.1, 1), lambda: layer.dropout_bwd(x, n, 0.1, 1),
                 lambda: layer.qk_norm_rope(q, None, None, None, None, n),
                 lambda: layer.qk_norm_rope_bwd(q, None, q, None, None, None, None, n),
                 lambda: layer.gated_ffn(x, w, w, Shaped.of((64, 72)), n),
                 lambda: layer.gated_ffn_bwd(x, x, w, w, Shaped.of((64, 72)), n),
                 lambda: layer.gated_ffn_workspace_bytes(n, 64, 72)):
        with pytest.raises(ValueError, match="at most 2147483647"):
            call()


@pytest.mark.parametrize("n", (2 ** 31, 2 ** 32 + 8))
def test_widths_past_32_bits_are_refused(n, device):
    x = Shaped.of((1, n))
    wide, tall, q = Shaped.of((8, n)), Shaped.of((n, 8)), Shaped.of((1, n, 8))
    for call in (lambda: layer.dropout_add(x, 1, 0.1, 1), lambda: layer.dropout_bwd(x, 1, 0.1, 1),
                 lambda: layer.qk_norm_rope(q, None, None, None, None, 1),
                 lambda: layer.qk_norm_rope(Shaped.of((1, 1, n)), None, None, None, None, 1),
                 lambda: layer.qk_norm_rope(Shaped.of((1, 1, 8)), q, None, None, None, 1),
                 lambda: layer.gated_ffn(x, wide, wide, tall, 1),
                 lambda: layer.gated_ffn(Shaped.of((1, 8)), tall, tall, wide, 1),
                 lambda: layer.gated_ffn_workspace_bytes(1, n, 8), lambda: layer.gated_ffn_workspace_bytes(1, 8, n)):
        with pytest.raises(ValueError, match="at most 2147483647"):
            call()


class Here(torch.Tensor):
    """A host tensor that says it lies on the current device."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def _in(memory, dtype, *shape, at=0):
    """A tensor at byte `at` of `memory` (uint8)."""
    n = torch.empty(0, dtype=dtype).element_size()
    for s in shape:
        n *= s
    return memory[at:at + n].view(dtype).view(*shape).as_subclass(Here)


def _new(dtype, *shape):
    return torch.zeros(shape, dtype=dtype).as_subclass(Here)


BF, F4, I4 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.parametrize("name", ["row_ids", "x", "residual"])
def test_dropout_outputs_stand_apart(name, device):
    N, d = 64, 8
    m = torch.zeros(4096, dtype=torch.uint8)
    rows, x, res = _new(I4, N), _new(F4, N, d), _new(F4, N, d)
    out = _in(m, F4, N, d)
    rows, x, res = (_in(m, I4, N, at=64) if name == "row_ids" else rows, _in(m, F4, N, d, at=64) if name == "x" else x,
                    _in(m, F4, N, d, at=64) if name == "residual" else res)
    with pytest.raises(ValueError, match="overlaps"):
        layer.dropout_add(x, N, 0.1, 1, residual=res, row_ids=rows, out=out)
    if name != "residual":
        with pytest.raises(ValueError, match="overlaps"):
            layer.dropout_bwd(x, N, 0.1, 1, row_ids=rows, out=out)


QK_INS = ["q", "k", "q_weight", "k_weight", "inv_freq", "positions", "seq_id", "cu_seqlens", "first_pos", "err_flag"]


def _qk_ins(m, name, N):
    """The inputs of the head norms, `name` inside m."""
    shapes = dict(q=(F4, N, 2, 16), k=(F4, N, 1, 16), q_weight=(F4, 16), k_weight=(F4, 16), inv_freq=(F4, 8),
                  positions=(I4, N), seq_id=(I4, N), cu_seqlens=(I4, 3), first_pos=(I4, 2), err_flag=(I4, 1))
    if name != "positions":
        del shapes["positions"]
    return {n: _in(m, *s, at=64) if n == name else _new(*s) for n, s in shapes.items()}


@pytest.mark.parametrize("name", QK_INS)
def test_head_norm_outputs_stand_apart(name, device):
    N = 32
    m = torch.zeros(1 << 16, dtype=torch.uint8)
    v = _qk_ins(m, name, N)
    ins = [v.pop(n) for n in ("q", "k", "q_weight", "k_weight", "inv_freq")]
    for which, heads in (("q_out", 2), ("k_out", 1)):
        with pytest.raises(ValueError, match="overlaps"):
            layer.qk_norm_rope(*ins, N, **v, **{which: _in(m, F4, N, heads, 16)})


@pytest.mark.parametrize("name", QK_INS + ["dq_out", "dk_out"])
def test_head_norm_workspace_stands_apart(name, device):
    N = 32
    m = torch.zeros(1 << 16, dtype=torch.uint8)
    v = _qk_ins(m, name, N)
    ins = [v.pop(n) for n in ("q", "k", "q_weight", "k_weight", "inv_freq")]
    grads = [_in(m, F4, N, h, 16) if name == n else _new(F4, N, h, 16) for n, h in (("dq_out", 2), ("dk_out", 1))]
    with pytest.raises(ValueError, match="overlaps"):
        layer.qk_norm_rope_bwd(*grads, *ins, N, **v, workspace=m.as_subclass(Here))


@pytest.mark.parametrize("name", ["x", "w_gate", "w_up", "w_down", "out", "dy", "preact", "dw"])
def test_gated_ffn_workspace_stands_apart(name, device):
    N, d, f = 4, 8, 16
    m = torch.zeros(1 << 16, dtype=torch.uint8)
    at = lambda n, *s: _in(m, *s) if n == name else _new(*s)   # noqa: E731
    x, ws = at("x", BF, N, d), (at("w_gate", BF, f, d), at("w_up", BF, f, d), at("w_down", BF, d, f))
    if name not in ("dy", "preact", "dw"):
        with pytest.raises(ValueError, match="overlaps"):
            layer.gated_ffn(x, *ws, N, out=at("out", BF, N, d), workspace=m.as_subclass(Here))
    if name != "out":
        dw = (_new(F4, f, d), at("dw", F4, f, d), _new(F4, d, f))
        with pytest.raises(ValueError, match="overlaps"):
            layer.gated_ffn_bwd(at("dy", BF, N, d), x, *ws, N, preact=at("preact", F4, N, 2 * f), dw=dw,
                                workspace=m.as_subclass(Here))


def test_arguments_that_are_no_tensors_are_named(device):
    x, w, wd = _new(BF, 4, 8), _new(BF, 16, 8), _new(BF, 8, 16)
    for args, name in (((x, None, w, wd), "w_gate"), ((x, w, None, wd), "w_up"), ((x, w, w, [1.0]), "w_down"),
                       ((None, w, w, wd), "x")):
        with pytest.raises(TypeError, match=f"{name} must be a torch.Tensor"):
            layer.gated_ffn(*args, 4)
        with pytest.raises(TypeError, match=f"{name} must be a torch.Tensor"):
            layer.gated_ffn_bwd(x, *args, 4)
    with pytest.raises(TypeError, match="out must be a torch.Tensor"):
        layer.dropout_add(x, 4, 0.1, 1, out=[0.0])


def test_a_key_output_without_keys_is_refused(device):
    q = _new(BF, 4, 2, 16)
    with pytest.raises(ValueError, match="k_out"):
        layer.qk_norm_rope(q, None, None, None, None, 4, k_out=_new(BF, 4, 1, 16))
