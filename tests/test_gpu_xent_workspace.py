"""The head's loss in workspaces of exactly the size it asks for, for operands of every alignment: nothing behind them is touched, and
what was in them counts for nothing."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import api
from tests.test_gpu_xent_digits import _data, _reference
from tests.operator_bounds import within

pytestmark = pytest.mark.gpu

GUARD = 4096


def _shifted(t, by):
    room = torch.zeros(t.numel() + 16, dtype=t.dtype, device="cuda")
    out = room[by:by + t.numel()].view_as(t)
    return out.copy_(t)


def _workspace(need, fill):
    room = torch.full((need + GUARD,), fill, dtype=torch.uint8, device="cuda")
    return room, room[:need]


@pytest.mark.parametrize("dtype,code", [(torch.float32, 2), (torch.float16, 3), (torch.bfloat16, 6)])
@pytest.mark.parametrize("n,d,V", [(1, 512, 3000), (7, 63, 300), (40, 2048, 900), (300, 96, 2000), (4100, 16, 33000), (5000, 64, 21)])
@pytest.mark.parametrize("shift_h,shift_w", [(0, 0), (1, 0), (0, 1), (1, 3)])
def test_exact_workspaces(n, d, V, dtype, code, shift_h, shift_w):
    h, W, labels, up = _data(n, d, V, dtype, n + V)
    h, W = _shifted(h, shift_h), _shifted(W, shift_w)
    aligned = shift_h == shift_w == 0
    results = []
    for fill in (0, 255):  # (255: NaN in every type)
        need = api.ecc_xent_workspace_bytes(n, d, V, code, False, aligned)
        room, ws = _workspace(need, fill)
        loss, stats, counted = api.ecc_xent_fwd(h, W, labels, reduction="none", workspace=ws)
        back_need = api.ecc_xent_workspace_bytes(n, d, V, code, True, aligned)
        back_room, back = _workspace(back_need, fill)
        dh, dW = api.ecc_xent_bwd(h, W, labels, up, stats, counted, reduction="none", workspace=back)
        assert bool((room[need:] == fill).all()) and bool((back_room[back_need:] == fill).all())
        results.append((loss, dh, dW))
    assert all(torch.equal(a, c) for a, c in zip(*results))
    ref = _reference(h, W, labels, "none", up)
    for k, name in enumerate(("loss", "dhidden", "dweight")):
        within(results[0][k], ref[2 * k], ref[2 * k + 1], name)
    if aligned and d % 8 == 0:  # one byte fewer is refused
        for call, size in ((lambda ws: api.ecc_xent_fwd(h, W, labels, reduction="none", workspace=ws), need),
                           (lambda ws: api.ecc_xent_bwd(h, W, labels, up, stats, counted, reduction="none", workspace=ws), back_need)):
            with pytest.raises(api.EccError) as e:
                call(_workspace(size, 0)[1][:size - 1])
            assert e.value.status == -3


def test_more_tiles_than_one_launch_takes():
    """2^30 rows: two tiles of classes for each tile of rows would be a grid of 2^32 threads."""
    n, d, V = (1 << 30) + 300, 8, 200
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = torch.randn(V, d, generator=gen, device="cuda").to(torch.bfloat16)
    h = torch.empty(n, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    labels = torch.randint(0, V, (n,), generator=gen, device="cuda")
    loss = api.ecc_xent_fwd(h, W, labels, reduction="none", keep=False)[0]
    for part in (slice(0, 300), slice((1 << 29) - 150, (1 << 29) + 150), slice(n - 600, n)):
        ref = _reference(h[part], W, labels[part], "none", torch.ones(len(loss[part]), device="cuda"))
        within(loss[part], ref[0], ref[1], "loss")
    del h, labels, loss
    torch.cuda.empty_cache()
