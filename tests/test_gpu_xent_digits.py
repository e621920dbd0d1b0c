"""The linear head's loss and gradients against bounds of plain float32 arithmetic on the operands as they are: nothing in them knows
of the largest value of a tensor, of the number of rows, or of how the logits' gradient is held, but for what a type needs: 16-bit
types hold it to twice their bits, float16 as a multiple of 2^-39 of the largest upstream gradient."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import api
from paper_2510_20271_amd.loss import linear_cross_entropy
from tests.operator_bounds import E, rounding, within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
IGNORE = -100


def _lse_off(z, d):
    """How far the log-sum-exp of the last axis moves when every entry moves by up to d."""
    at = torch.logsumexp(z, 1, keepdim=True)
    return torch.maximum(torch.logsumexp(z + d, 1, keepdim=True) - at, at - torch.logsumexp(z - d, 1, keepdim=True))


def _reference(h, W, labels, reduction, up):
    """(loss, its bound, dh, its bound, dW, its bound) in float64."""
    dtype = h.dtype
    n, d = h.shape
    V = W.shape[0]
    keep = labels != IGNORE
    h, W = torch.where(keep[:, None], h, torch.zeros_like(h)).double(), W.double()
    at = torch.where(keep, labels, 0)[:, None]
    z = h @ W.t()
    # float32 sums of d products in some order
    d_z = (4 * math.sqrt(d) + 4) * E * (h.abs() @ W.abs().t())
    lse = torch.logsumexp(z, 1, keepdim=True)
    d_lse = _lse_off(z, d_z)
    # exponentials: an argument's rounding (|x| p <= log V over a row), an ulp or two each, their float32 sum
    rows = (lse - z.gather(1, at))[:, 0]
    d_rows = (d_lse + d_z.gather(1, at))[:, 0] + (16 + 2 * math.log(V + 1)) * E * (1 + rows.abs())
    zero = torch.zeros_like(rows)
    rows, d_rows = torch.where(keep, rows, zero), torch.where(keep, d_rows, zero)
    count = max(1, int(keep.sum()))
    by = {"mean": 1.0 / count, "sum": 1.0}.get(reduction)
    loss, d_loss = (rows, d_rows) if by is None else (rows.sum() * by, d_rows.sum() * by)
    d_loss = d_loss + 4 * E * loss.abs() + 1e-30
    g = up.double() if by is None else torch.full_like(rows, float(up) * by)
    g = torch.where(keep, g, zero)[:, None]
    hit = torch.zeros_like(z).scatter_(1, at, 1.0)
    p = torch.exp(z - lse)
    # one minus the label's probability, from the others' sum
    others = torch.logsumexp(z.masked_fill(hit.bool(), -math.inf), 1, keepdim=True) - z.gather(1, at)
    miss = torch.sigmoid(others)
    d_others = _lse_off(z.masked_fill(hit.bool(), -math.inf), d_z) + d_z.gather(1, at)
    d_miss = miss * torch.expm1((d_others + (16 + 2 * math.log(V + 1)) * E).clamp_max(50.0)).clamp_max(1.0)
    off = d_z + d_lse + 8 * E * (1 + (z - lse).abs())
    d_p = torch.exp((z - lse + off).clamp_max(0.0)) - p + 4 * E * p + 4 * 2.0 ** -126 * (p > 0)
    dz = torch.where(hit.bool(), -miss, p) * g
    d_dz = torch.where(hit.bool(), d_miss + 4 * E * miss, d_p) * g.abs()
    half = 0.0 if dtype == F32 else (torch.finfo(dtype).eps / 2) ** 2
    d_dz = d_dz + (half + E) * dz.abs()
    if dtype == F16:
        d_dz = d_dz + 2.0 ** -39 * g.abs().max() * (g != 0)
    dh, dW = dz @ W, dz.t() @ h
    d_dh = d_dz @ W.abs() + (4 * math.sqrt(V) + 8) * E * (dz.abs() @ W.abs()) + rounding(dh, dtype) + 2.0 ** -149
    d_dW = d_dz.t() @ h.abs() + (4 * math.sqrt(n) + 8) * E * (dz.abs().t() @ h.abs()) + rounding(dW, dtype) + 2.0 ** -149
    return loss, d_loss, dh, d_dh, dW, d_dW


def _check(h, W, labels, reduction, up):
    hr, Wr = h.clone().requires_grad_(True), W.clone().requires_grad_(True)
    loss = linear_cross_entropy(hr, Wr, labels, reduction=reduction)
    dh, dW = torch.autograd.grad(loss, (hr, Wr), up)
    ref = _reference(h, W, labels, reduction, up)
    within(loss.detach(), ref[0], ref[1], "loss")
    within(dh, ref[2], ref[3], "dhidden")
    within(dW, ref[4], ref[5], "dweight")


def _data(n, d, V, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = torch.randn(V, d, generator=gen, device="cuda") * d ** -0.5
    labels = torch.randint(0, V, (n,), generator=gen, device="cuda")
    h = 2 * torch.randn(n, d, generator=gen, device="cuda") + 8 * torch.rand(n, 1, generator=gen, device="cuda") * W[labels]
    if n > 1:
        labels[torch.rand(n, generator=gen, device="cuda") < 0.1] = IGNORE
    return h.to(dtype), W.to(dtype), labels, 0.5 + torch.rand(n, generator=gen, device="cuda")


# 16-bit types: each way that the logits' gradient takes (made in a product's epilogue, or from split sums: long rows of features, up to
# 1024 classes), on both sides of every rule on the number of rows, and each tile
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,d,V", [(1, 64, 3000), (8, 64, 3000), (8, 2048, 600), (64, 40, 700), (65, 40, 700), (65, 2048, 600),
                                   (300, 96, 40), (520, 264, 300), (4099, 64, 21), (2300, 520, 2304), (4100, 16, 33000)])
@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_gradients_of_16_bit_heads(n, d, V, dtype, reduction):
    h, W, labels, up = _data(n, d, V, dtype, n + d + V)
    _check(h, W, labels, reduction, up if reduction == "none" else torch.tensor(0.75, device="cuda"))


WIDE = [(100, 512, 2000), (128, 256, 700), (129, 512, 5000), (300, 512, 2000), (300, 511, 2000), (4097, 300, 250)]


@pytest.mark.parametrize("n,d,V", WIDE)
@pytest.mark.parametrize("low", [-1e6, -1e9, -1e30, -torch.finfo(torch.float32).max])
def test_float32_with_a_masked_class(n, d, V, low):
    """A finite weight that masks its class, at a feature that every row has."""
    h, W, labels, up = _data(n, d, V, F32, n + V)
    h[:, 0] = 1.0
    W[5] = 0.0
    W[5, 0] = low
    labels[labels == 5] = 6
    _check(h, W, labels, "mean", torch.tensor(0.75, device="cuda"))


@pytest.mark.parametrize("n,d,V", WIDE)
@pytest.mark.parametrize("power", [24, 32, 40, 60])
def test_float32_with_one_large_row(n, d, V, power):
    """One row of features far above the others, as a sample that diverged leaves it."""
    h, W, labels, up = _data(n, d, V, F32, n + V)
    h[n // 2] *= 2.0 ** power
    _check(h, W, labels, "none", up)


@pytest.mark.parametrize("n,d,V", WIDE)
def test_float32_with_features_and_classes_of_many_sizes(n, d, V):
    """Features of sizes from 1e6 to 1e-6 with weights of the inverse sizes, classes from 1 to 1e-6."""
    h, W, labels, up = _data(n, d, V, F32, n + V)
    by = 10.0 ** -(torch.arange(d, device="cuda") % 13 - 6).float()
    W = W * 10.0 ** -(torch.arange(V, device="cuda") % 7).float()[:, None]
    _check(h * by, W / by, labels, "mean", torch.tensor(0.75, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,V", WIDE)
def test_upstream_gradients_of_many_sizes(n, d, V, dtype):
    """From 1 to 1e-8 a row: each row of hidden's gradient to its own size."""
    h, W, labels, up = _data(n, d, V, dtype, n + V)
    _check(h, W, labels, "none", up * 10.0 ** -(torch.arange(n, device="cuda") % 9).float())


def test_rows_do_not_depend_on_how_many_there_are():
    """128 rows alone and among 300, one of them large: the same losses to a plain product's rounding."""
    h, W, labels, up = _data(300, 512, 2000, F32, 1)
    h[200] *= 2.0 ** 40
    few = api.ecc_xent_fwd(h[:128].contiguous(), W, labels[:128].contiguous(), reduction="none")[0]
    all_rows = api.ecc_xent_fwd(h, W, labels, reduction="none")[0]
    bound = _reference(h[:128], W, labels[:128], "none", up[:128])[1]
    assert bool(((few - all_rows[:128]).abs().double() <= 2 * bound).all())


# hidden's gradient and the weight's straight from their products, from split sums, and from several pieces of the classes
@pytest.mark.parametrize("n,d,V", [(41, 20, 30), (9, 64, 5000), (300, 512, 2000), (4100, 16, 33000), (5000, 64, 21)])
@pytest.mark.parametrize("up", [1.3 * 2.0 ** -126, 1.7 * 2.0 ** -120, 0.75, 1.3 * 2.0 ** 100])
def test_float32_upstream_gradients_of_any_size(n, d, V, up):
    """A mean's upstream gradient over a count that is no power of two: their quotient may have no digits of its own where the gradients
    have all of theirs."""
    h, W, labels, _ = _data(n, d, V, F32, n + V)
    labels[0] = 1
    far = 2.0 ** 40 if up < 1e-30 else 2.0 ** -40  # (logits are the same)
    up = torch.tensor(up, device="cuda")
    for by in (1.0, far, 1.0 / far):
        hr, Wr = (h * by).requires_grad_(True), (W / by).requires_grad_(True)
        loss = linear_cross_entropy(hr, Wr, labels)
        grads = torch.autograd.grad(loss, (hr, Wr), up)
        ref = _reference(hr.detach(), Wr.detach(), labels, "mean", up)
        within(loss.detach(), ref[0], ref[1], "loss")
        for got, want, bound, name in zip(grads, ref[2::2], ref[3::2], ("dhidden", "dweight")):
            beyond = want.abs() + bound > torch.finfo(F32).max  # (features of 1e12 and an upstream gradient of 1e30)
            assert bool((got[want.abs() - bound > torch.finfo(F32).max].abs() == math.inf).all())
            within(torch.where(beyond, 0.0, got), torch.where(beyond, 0.0, want), bound, name)
