"""Group norm with an activation against its plain form in 64 bits: shapes, types, activations, gradients, edges."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import api
from paper_2510_20271_amd.norm import GroupNormAct, group_norm_act
from tests.operator_bounds import E, norm_reference, within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SHAPES = [  # batch, points, channels, groups
    (1, 1, 1, 1), (1, 1, 8, 8), (2, 1, 6, 2), (3, 5, 7, 7), (1, 64, 32, 8), (2, 63, 30, 5), (5, 17, 181, 1), (1, 129, 24, 3),
    (65, 1, 128, 8), (1, 4099, 4, 2), (2, 1500, 64, 32), (1, 20000, 48, 6), (3, 700, 320, 32), (1, 3, 8192, 4),
    (2, 9, 1500, 3), (1, 70001, 3, 1), (7, 333, 33, 11), (1, 31, 2050, 1), (300, 50, 16, 4), (1, 1, 65536, 16),
]


def _data(shape, groups, dtype, seed=0, offset=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, S, C = shape
    x = torch.randn(N, S, C, generator=gen, device="cuda") * 1.5 + torch.randn(C, generator=gen, device="cuda") + offset
    dy = torch.randn(N, S, C, generator=gen, device="cuda")
    w = 1 + 0.3 * torch.randn(C, generator=gen, device="cuda")
    b = 0.3 * torch.randn(C, generator=gen, device="cuda")
    return x.to(dtype), dy.to(dtype), w, b


def _check(x, groups, w, b, act, dy, eps=1e-5):
    leaves = [t.clone().requires_grad_(True) if t is not None else None for t in (x, w, b)]
    y = group_norm_act(leaves[0], groups, leaves[1], leaves[2], eps=eps, act=act)
    got = torch.autograd.grad(y, [t for t in leaves if t is not None], dy)
    C = x.shape[-1]
    flat = (x.shape[0], x.numel() // x.shape[0] // C, C)
    y_, dy_, dx, d_dx, dw, d_dw, db, d_db = norm_reference(x.reshape(flat), groups, w, b, eps, act, dy.reshape(flat))
    assert y.dtype == x.dtype and got[0].dtype == x.dtype
    within(y.detach().reshape(flat), y_, dy_, "y")
    within(got[0].reshape(flat), dx, d_dx, "dx")
    if w is not None:
        within(got[1], dw, d_dw, "dweight")
    if b is not None:
        within(got[-1], db, d_db, "dbias")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("N,S,C,G", SHAPES)
def test_against_the_plain_form(N, S, C, G, dtype):
    x, dy, w, b = _data((N, S, C), G, dtype, seed=N + S + C)
    _check(x, G, w, b, "silu", dy)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(2, 300, 24, 4), (1, 30000, 40, 5), (2, 7, 9, 3)])
def test_activations_and_missing_parameters(N, S, C, G, dtype, act):
    x, dy, w, b = _data((N, S, C), G, dtype, seed=5)
    _check(x, G, w, b, act, dy)
    _check(x, G, w, None, act, dy)
    _check(x, G, None, None, act, dy)


@pytest.mark.parametrize("N,S,C,G", [(2, 300, 24, 4), (1, 50000, 32, 4), (1, 200001, 6, 2)])
def test_offsets_far_above_the_spread(N, S, C, G):
    """Squares are summed about a value of the data: a mean of 1000 spreads costs no digits but those of x itself."""
    x, dy, w, b = _data((N, S, C), G, F32, seed=6, offset=1500.0)
    _check(x, G, w, b, "silu", dy)


@pytest.mark.parametrize("where", ["first", "last"])
@pytest.mark.parametrize("N,S,C,G", [(1, 640, 16, 2), (1, 60000, 16, 2)])
def test_one_value_far_from_the_rest(N, S, C, G, where):
    x, dy, w, b = _data((N, S, C), G, F32, seed=7)
    x[0, 0 if where == "first" else -1, 0] = 3e4
    _check(x, G, w, b, "none", dy)


def test_equal_values():
    """No spread at all: the variance is 0 to the bit, y is act(bias) and the scale 1 / sqrt(eps)."""
    for S in (1, 40, 30000):
        x = torch.full((2, S, 12), 3.25, device="cuda")
        b = torch.linspace(-1, 1, 12, device="cuda")
        y, stats = api.ecc_norm_fwd(x, 3, None, b, act="relu")
        assert torch.equal(y, b.clamp_min(0).expand_as(y))
        assert torch.equal(stats[..., 0], torch.full((2, 3), 3.25, device="cuda", dtype=torch.float64))
        assert float((stats[..., 1] * float(np.float32(1e-5)) ** 0.5 - 1).abs().max()) < 1e-12
        y, _ = api.ecc_norm_fwd(x, 3, None, b, eps=0.0)  # 0 / 0
        assert bool(torch.isnan(y).all())


@pytest.mark.parametrize("S", [20, 40000])
def test_nan_and_inf_spoil_their_own_group(S):
    x, dy, w, b = _data((2, S, 12), 3, F32, seed=8)
    want, stats = api.ecc_norm_fwd(x, 3, w, b)
    ref = api.ecc_norm_bwd(x, dy, 3, stats, w, b)
    for bad in (float("nan"), float("inf")):
        z = x.clone()
        z[1, S // 2, 5] = bad
        y, stats = api.ecc_norm_fwd(z, 3, w, b)
        assert bool(torch.isnan(y[1, :, 4:8]).all())
        assert torch.equal(y[0], want[0]) and torch.equal(y[1, :, :4], want[1, :, :4]) and torch.equal(y[1, :, 8:], want[1, :, 8:])
        gx, gw, gb = api.ecc_norm_bwd(z, dy, 3, stats, w, b)
        assert torch.equal(gx[0], ref[0][0]) and torch.equal(gx[1, :, 8:], ref[0][1, :, 8:])
        assert bool(torch.isnan(gw[4:8]).all()) and torch.equal(gw[8:], ref[1][8:]) and torch.equal(gb[:4], ref[2][:4])


def test_extreme_activations_stay_finite():
    b = torch.tensor([-1e4, -100.0, -88.5, 88.5, 100.0, 1e4], device="cuda")
    x = torch.randn(1, 50, 6, device="cuda", generator=torch.Generator("cuda").manual_seed(0))
    _check(x, 6, torch.ones(6, device="cuda"), b, "silu", torch.ones_like(x))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layouts_of_the_grid(dtype):
    """[batch, D, H, W, channels], [batch, channels]; a view with other strides, a slice off its alignment."""
    x, dy, w, b = _data((2, 3 * 5 * 7, 12), 4, dtype, seed=9)
    _check(x.view(2, 3, 5, 7, 12), 4, w, b, "silu", dy.view(2, 3, 5, 7, 12))
    _check(x[:, 0], 4, w, b, "silu", dy[:, 0])
    first = x.permute(0, 2, 1).contiguous()  # channels first in memory
    assert torch.equal(group_norm_act(first.permute(0, 2, 1), 4, w, b), group_norm_act(x, 4, w, b))
    room = torch.empty(x.numel() + 3, dtype=dtype, device="cuda")
    for shift in (1, 2, 3):
        off = room[shift:shift + x.numel()].view_as(x)
        off.copy_(x)
        _check(off, 4, w, b, "silu", dy)
        out = torch.full((x.numel() + 8,), 7.0, dtype=dtype, device="cuda")
        api.ecc_norm_fwd(off, 4, w, b, y=out[shift:shift + x.numel()].view_as(x))
        assert bool((out[:shift] == 7).all()) and bool((out[shift + x.numel():] == 7).all())


def test_same_bits_again_and_parts_of_the_gradients():
    for shape, G in (((4, 100, 24), 4), ((1, 90000, 24), 4)):
        x, dy, w, b = _data(shape, G, F32, seed=10)
        y, stats = api.ecc_norm_fwd(x, G, w, b)
        full = api.ecc_norm_bwd(x, dy, G, stats, w, b)
        for _ in range(3):
            y2, stats2 = api.ecc_norm_fwd(x, G, w, b)
            assert torch.equal(y, y2) and torch.equal(stats, stats2)
            for a, c in zip(full, api.ecc_norm_bwd(x, dy, G, stats, w, b)):
                assert torch.equal(a, c)
        assert torch.equal(api.ecc_norm_fwd(x, G, w, b, keep=False)[0], y)
        names = ("grad_x", "grad_weight", "grad_bias")
        for skip in (names[:1], names[1:], names[:2], names[2:], names[1:2]):
            for name, a, c in zip(names, full, api.ecc_norm_bwd(x, dy, G, stats, w, b, skip=skip)):
                assert (c is None) if name in skip else torch.equal(a, c)


def test_gradient_against_differences():
    """Central differences of the float64 plain form at a step of 1e-4: their error is 1e-8 of third derivatives."""
    x, dy, w, b = _data((1, 6, 4), 2, F32, seed=11)
    xr = x.clone().requires_grad_(True)
    group_norm_act(xr, 2, w, b).backward(dy)
    for s, c in ((0, 0), (3, 2), (5, 3)):
        d = []
        for sign in (1, -1):
            z = x.double().clone()
            z[0, s, c] += sign * 1e-4
            d.append(float((norm_reference(z, 2, w, b, 1e-5, "silu")[0] * dy.double()).sum()))
        assert abs((d[0] - d[1]) / 2e-4 - float(xr.grad[0, s, c])) < 1e-4


def test_module_and_empty_inputs():
    layer = GroupNormAct(4, 16, act="relu").cuda()
    x = torch.randn(2, 5, 6, 16, device="cuda", generator=torch.Generator("cuda").manual_seed(1), requires_grad=True)
    layer(x).sum().backward()
    assert layer.weight.grad.shape == (16,) and x.grad.shape == x.shape
    half = layer(x.detach().bfloat16())
    assert half.dtype == BF16
    for shape in ((0, 4, 16), (2, 0, 16)):
        e = torch.zeros(shape, device="cuda", requires_grad=True)
        out = layer(e)
        assert out.shape == shape
        layer.zero_grad()
        out.sum().backward()
        assert e.grad.shape == shape and bool((layer.weight.grad == 0).all())
    with torch.no_grad():
        assert torch.equal(layer(x), layer(x.detach()))


def test_on_a_stream_of_its_own_and_in_graphs():
    x, dy, w, b = _data((2, 9000, 24), 4, F32, seed=12)
    y, stats = api.ecc_norm_fwd(x, 4, w, b)
    want = (y, *api.ecc_norm_bwd(x, dy, 4, stats, w, b))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, st2 = api.ecc_norm_fwd(x, 4, w, b)
        got = (y2, *api.ecc_norm_bwd(x, dy, 4, st2, w, b))
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    ins = [x.clone(), x.clone()]
    graphs, outs = [], []
    for xi in ins:  # two graphs: neither may use the other's workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            yi, st = api.ecc_norm_fwd(xi, 4, w, b)
            outs.append((yi, *api.ecc_norm_bwd(xi, dy, 4, st, w, b)))
        graphs.append(g)
    side = torch.cuda.Stream()
    for k in range(4):
        for i, xi in enumerate(ins):
            xi.copy_(_data((2, 9000, 24), 4, F32, seed=20 + 2 * k + i)[0])
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for xi, out in zip(ins, outs):
            ye, st = api.ecc_norm_fwd(xi, 4, w, b)
            for a, c in zip((ye, *api.ecc_norm_bwd(xi, dy, 4, st, w, b)), out):
                assert torch.equal(a, c)


def test_refusals():
    x = torch.zeros(2, 5, 12, device="cuda")
    w = torch.ones(12, device="cuda")
    for call in (lambda: group_norm_act(x.cpu(), 3), lambda: group_norm_act(x, 5), lambda: group_norm_act(x, 0),
                 lambda: group_norm_act(x, 3, act="tanh"), lambda: group_norm_act(x.double(), 3),
                 lambda: group_norm_act(x, 3, w[:6]), lambda: group_norm_act(x[0, 0], 3),
                 lambda: api.ecc_norm_fwd(x.transpose(0, 1), 3), lambda: api.ecc_norm_fwd(x, 3, w.double()),
                 lambda: api.ecc_norm_fwd(x, 3, y=torch.zeros(2, 5, 11, device="cuda")),
                 lambda: api.ecc_norm_bwd(x, x.half(), 3, torch.zeros(2, 3, 2, dtype=torch.float64, device="cuda")),
                 lambda: api.ecc_norm_bwd(x, x, 3, torch.zeros(2, 3, 2, device="cuda")),
                 lambda: GroupNormAct(3, 12).cuda()(x[..., :6])):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: api.ecc_norm_fwd(x, 5), -1), (lambda: api.ecc_norm_fwd(x, 3, eps=-1.0), -1),
                         (lambda: api.ecc_norm_fwd(x, 3, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), -3)):
        with pytest.raises(api.EccError) as e:
            call()
        assert e.value.status == status


def test_features_beyond_32_bits():
    """2.15e9 features in one item: statistics over all of them, the last points' outputs and gradients."""
    S, C, G = (1 << 25) + 5, 64, 8
    gen = torch.Generator(device="cuda").manual_seed(16)
    x = torch.empty(1, S, C, dtype=BF16, device="cuda").normal_(generator=gen)
    dy = torch.empty(1, S, C, dtype=BF16, device="cuda").normal_(generator=gen)
    w = 1 + 0.3 * torch.randn(C, generator=gen, device="cuda")
    b = 0.3 * torch.randn(C, generator=gen, device="cuda")
    y, stats = api.ecc_norm_fwd(x, G, w, b)
    gx, gw, gb = api.ecc_norm_bwd(x, dy, G, stats, w, b)
    part, m = 1 << 21, S * (C // G)

    def over(f):
        total = 0.0
        for r in range(0, S, part):
            total = total + f(x[0, r:r + part].double(), dy[0, r:r + part].double())
        return total

    def spread(t):
        return t.repeat_interleave(C // G)
    mean = over(lambda a, d: a.sum(0)).view(G, -1).sum(1) / m
    rstd = 1 / torch.sqrt(over(lambda a, d: ((a - spread(mean)) ** 2).sum(0)).view(G, -1).sum(1) / m + 1e-5)
    assert float((stats[0, :, 0] - mean).abs().max()) < 1e-6 and float((stats[0, :, 1] / rstd - 1).abs().max()) < 1e-6

    def terms(a, d):
        xhat = (a - spread(mean)) * spread(rstd)
        v = xhat * w + b
        s = torch.sigmoid(v)
        return xhat, v * s, d * s * (1 + v * (1 - s))
    db = over(lambda a, d: terms(a, d)[2].sum(0))
    dw = over(lambda a, d: (terms(a, d)[2] * terms(a, d)[0]).sum(0))
    # 2^31 / 64 terms of size 1 with random signs: sums of about 6e3, off by 300 E of the 3e7 terms' sizes at most
    assert float((gb - db).abs().max()) < 300 * E * S and float((gw - dw).abs().max()) < 300 * E * S
    xhat, want, dv = terms(x[0, -100:].double(), dy[0, -100:].double())
    assert bool(((y[0, -100:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all())
    m1 = spread((db * w).view(G, -1).sum(1) / m)
    m2 = spread((dw * w).view(G, -1).sum(1) / m)
    want = spread(rstd) * (dv * w - m1 - xhat * m2)
    assert bool(((gx[0, -100:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())


def test_refusals_of_empty_features():
    x = torch.zeros(0, 5, 12, device="cuda")
    for call in (lambda: group_norm_act(x, 3, act="tanh"), lambda: group_norm_act(x.int(), 3),
                 lambda: group_norm_act(x, 3, torch.ones(12))):
        with pytest.raises(ValueError):
            call()


def test_more_items_than_a_launch_takes():
    """Curves of eight thresholds: a block an item, in several launches."""
    n, T = 2 ** 25 + 70000, 8
    gen = torch.Generator("cuda").manual_seed(40)
    x = torch.randn(n, T, generator=gen, device="cuda", dtype=BF16)
    dy = torch.randn(n, T, generator=gen, device="cuda", dtype=BF16)
    w, b = 1 + torch.rand(T, generator=gen, device="cuda"), torch.rand(T, generator=gen, device="cuda")
    y, stats = api.ecc_norm_fwd(x, 2, w, b, act="none")
    dx, dw, db = api.ecc_norm_bwd(x, dy, 2, stats, w, b, act="none")
    for at in (0, 2 ** 24 - 50, 2 ** 25 - 50, n - 100):
        _, st = api.ecc_norm_fwd(x[at:at + 100].contiguous(), 2, w, b, act="none")
        some = api.ecc_norm_bwd(x[at:at + 100].contiguous(), dy[at:at + 100].contiguous(), 2, st, w, b, act="none")
        assert torch.equal(stats[at:at + 100], st) and torch.equal(dx[at:at + 100], some[0])
        assert torch.equal(y[at:at + 100], api.ecc_norm_fwd(x[at:at + 100].contiguous(), 2, w, b, act="none")[0])
    want_w, want_b, size_w, size_b = (torch.zeros(T, device="cuda", dtype=torch.float64) for _ in range(4))
    for k in range(0, n, 2 ** 22):
        g = dy[k:k + 2 ** 22].double()
        st = stats[k:k + 2 ** 22].repeat_interleave(T // 2, 1)
        t = g * (x[k:k + 2 ** 22].double() - st[..., 0]) * st[..., 1]
        want_w += t.sum(0); want_b += g.sum(0); size_w += t.abs().sum(0); size_b += g.abs().sum(0)
    # (a row's term is float32: a few roundings; the rows' sums are float64)
    assert bool(((dw.double() - want_w).abs() <= 2.0 ** -21 * size_w).all())
    assert bool(((db.double() - want_b).abs() <= 2.0 ** -21 * size_b).all())
