"""GPU: rows of a preference call that no sequence holds (a batch padded to a fixed count of rows).  They have log-probs
and a zero gradient, whatever they hold: values that are not finite there reach no other row, neither gradient nor loss,
and raise nothing."""
import pytest
import torch

from objective_util import F4, matrices
from paper_2606_29758_amd import objective

pytestmark = pytest.mark.gpu
I4, NAN, INF = torch.int32, float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    objective.load()


# one pass over the head with its gradient from LDS and from registers, float32 logits, tiles, rows by waves, chains
SIZES = [(12, 64, 300), (40, 136, 1000), (30, 3592, 200), (150, 64, 1000), (300, 1096, 60001), (2100, 64, 500)]


@pytest.mark.parametrize("many", [False, True])   # the pairs' step in one work-group, or by its own kernels
@pytest.mark.parametrize("N,d,V", SIZES)
def test_nothing_of_them_reaches_the_others(N, d, V, many):
    h, w, target = matrices(N, d, V, seed=N)
    g = torch.Generator("cuda").manual_seed(1)
    ref, weight = -5 - torch.rand(N, device="cuda", generator=g), 1 + torch.rand(N, device="cuda", generator=g)
    first, last, mid = 2, N - 3, N // 2
    cu = torch.tensor([first, mid, mid, last], dtype=I4, device="cuda")
    P = 2 ** 17 if many else 1
    chosen, rejected = torch.zeros(P, dtype=I4, device="cuda"), torch.full((P,), 2, dtype=I4, device="cuda")
    outside = torch.tensor([0, 1, N - 3, N - 2, N - 1], device="cuda")
    kw = dict(beta=0.1, loss_scale=1.0 / P, kind="sigmoid", temperature=0.7)

    def call(h, ref, weight, **more):
        err = torch.zeros(1, dtype=I4, device="cuda")
        o = objective.preference_loss(h, w, target, cu, chosen, rejected, N, logp_ref=ref, weight=weight, err_flag=err, **kw,
                                      **more)
        return o, int(err)

    want, err = call(h, ref, weight)
    assert err == 0 and want["loss"].isfinite() and want["d_w_head"].isfinite().all() and want["d_hidden"][first:last].any()
    assert not want["d_hidden"][outside].any()
    spoiled_h, spoiled_ref, spoiled_weight = h.clone(), ref.clone(), weight.clone()
    spoiled_h[0], spoiled_h[N - 2], spoiled_h[N - 1, 3] = NAN, INF, -INF
    spoiled_ref[1], spoiled_ref[N - 3], spoiled_weight[1] = NAN, -INF, INF
    for x, r, wt in ((spoiled_h, ref, weight), (h, spoiled_ref, spoiled_weight), (spoiled_h, spoiled_ref, spoiled_weight)):
        o, err = call(x, r, wt)
        assert err == 0
        for n in ("loss", "seq_ratio", "margin", "d_hidden", "d_w_head"):
            assert torch.equal(o[n], want[n]), n
        assert torch.equal(o["logp_new"][first:last], want["logp_new"][first:last])
        assert torch.equal(o["logp_new"][outside].isfinite(), x[outside].isfinite().all(1))
        one, err = call(x, r, wt, want_hidden=False, d_w_head=torch.full((V, d), NAN, dtype=F4, device="cuda"))
        assert err == 0 and one["d_w_head"].isfinite().all()
        none, err = call(x, r, wt, want_hidden=False, want_head=False)
        assert err == 0 and none["loss"].isfinite()


@pytest.mark.parametrize("N", [12, 40, 150, 2100])
def test_rows_of_a_sequence_still_raise_the_bit(N):
    """Also those of a sequence that stands in no pair."""
    h, w, target = matrices(N, 64, 300, seed=N)
    cu = torch.tensor([0, N // 3, N // 2, N], dtype=I4, device="cuda")
    pair = torch.tensor([0], dtype=I4, device="cuda"), torch.tensor([1], dtype=I4, device="cuda")
    ref = torch.zeros(N, device="cuda")
    for row in (1, N - 1):
        for spoil in ("h", "ref"):
            x, r = h.clone(), ref.clone()
            (x if spoil == "h" else r)[row] = NAN
            for grads in (True, False):
                err = torch.zeros(1, dtype=I4, device="cuda")
                objective.preference_loss(x, w, target, cu, *pair, N, 0.1, 1.0, logp_ref=r, err_flag=err, want_hidden=grads,
                                          want_head=grads)
                assert int(err) == 16, (row, spoil, grads)
