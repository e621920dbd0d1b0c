"""Normalisations of so many items that the launches which join their groups would have more threads than a grid may have."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import api
from tests.operator_bounds import E, norm_reference, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,points,channels,groups", [
    (140000, 1096, 30, 30),          # 4.2e6 groups: blocks of 1024 threads each in the backward pass
    ((1 << 21) + 5, 1, 1026, 2),     # curves: groups wider than a block, two column ranges a row
])
def test_more_groups_than_one_launch_joins(batch, points, channels, groups):
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty(batch, points, channels, dtype=torch.float16, device="cuda").normal_(generator=gen)
    dy = torch.empty_like(x).normal_(generator=gen)
    w = 1 + 0.2 * torch.randn(channels, generator=gen, device="cuda")
    b = 0.2 * torch.randn(channels, generator=gen, device="cuda")
    y, stats = api.ecc_norm_fwd(x, groups, w, b, act="none")
    dx, dw, db = api.ecc_norm_bwd(x, dy, groups, stats, w, b, act="none")
    last = (1 << 21) // max(1, points)  # items around what one launch takes, and the ends
    for part in (slice(0, 3), slice(batch // 2 - 2, batch // 2 + 2), slice(max(0, last - 2), last + 2), slice(batch - 4, batch)):
        ref = norm_reference(x[part], groups, w, b, 1e-5, "none", dy[part])
        within(y[part], ref[0], ref[1], "y")
        within(dx[part], ref[2], ref[3], "dx")
    # the parameters' gradients: every item's
    want = torch.zeros(2, channels, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    Cg, step = channels // groups, max(1, (1 << 26) // (points * channels))
    for n in range(0, batch, step):
        xd, d = x[n:n + step].double(), dy[n:n + step].double()
        g = xd.view(len(xd), points, groups, Cg)
        mean = g.mean((1, 3), keepdim=True)
        xhat = ((g - mean) / torch.sqrt(((g - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5)).view_as(xd)
        for k, t in enumerate((d, d * xhat)):
            want[k] += t.sum((0, 1))
            size[k] += t.abs().sum((0, 1))
    # shares of a block in float32 (300 E of their sizes), xhat to 224 E, the rest in float64
    assert bool(((db.double() - want[0]).abs() <= 300 * E * size[0] + E * want[0].abs()).all())
    assert bool(((dw.double() - want[1]).abs() <= 600 * E * (size[1] + size[0])).all())
