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
