"""Rows that are left out of the head's loss get zeros, whatever the weights and the upstream gradient hold."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import api
from tests.test_gpu_xent_digits import IGNORE, _data

pytestmark = pytest.mark.gpu


# hidden's gradient straight from its product, from split sums, and from several pieces of the classes
@pytest.mark.parametrize("n,d,V", [(40, 20, 30), (9, 64, 5000), (300, 96, 2000), (4100, 16, 33000), (5000, 64, 21)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_zeros_beside_weights_and_gradients_that_are_not_finite(n, d, V, dtype):
    h, W, labels, up = _data(n, d, V, dtype, n + V)
    labels[1:4] = IGNORE
    labels[0] = 1
    out = labels == IGNORE
    for bad in (float("-inf"), float("inf"), float("nan")):
        weight = W.clone()
        weight[5 % V, 2] = bad
        loss, stats, counted = api.ecc_xent_fwd(h, weight, labels, reduction="none")
        assert bool((loss[out] == 0).all())
        dh, _ = api.ecc_xent_bwd(h, weight, labels, up, stats, counted, reduction="none")
        assert bool((dh[out] == 0).all())
        for reduction in ("mean", "sum"):
            loss, stats, counted = api.ecc_xent_fwd(h, W, labels, reduction=reduction)
            dh, _ = api.ecc_xent_bwd(h, W, labels, torch.tensor(bad, device="cuda"), stats, counted, reduction=reduction)
            assert bool((dh[out] == 0).all()) and not bool(torch.isfinite(dh[~out]).any())
