"""Refusals of the normalisation's and the loss's entry points, made on the host before any GPU call (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd import _lib
from paper_2510_20271_amd.loss import LinearCrossEntropy, linear_cross_entropy
from paper_2510_20271_amd.norm import GroupNormAct, group_norm_act

FAKE = ctypes.c_void_p(0x1000)  # non-NULL, 256-aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def _norm(**kw):
    a = dict(x=FAKE, batch=2, points=9, channels=12, groups=3, dtype=2, weight=FAKE, bias=FAKE, eps=1e-5, act=2, y=FAKE,
             stats=FAKE, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return a


def _norm_fwd(a):
    return _lib.load().ecc_norm_fwd(a["x"], a["batch"], a["points"], a["channels"], a["groups"], a["dtype"], a["weight"],
                                    a["bias"], a["eps"], a["act"], a["y"], a["stats"], a["ws"], a["ws_bytes"], None)


def _norm_bwd(a, gy=FAKE, gx=FAKE, gw=FAKE, gb=FAKE):
    return _lib.load().ecc_norm_bwd(a["x"], gy, a["batch"], a["points"], a["channels"], a["groups"], a["dtype"], a["weight"],
                                    a["bias"], a["act"], a["stats"], gx, gw, gb, a["ws"], a["ws_bytes"], None)


NORM_BOTH = [
    (dict(x=None), INVALID, "x is"), (dict(batch=0), INVALID, "batch"), (dict(points=0), INVALID, "points"),
    (dict(channels=0), INVALID, "channels"), (dict(channels=1 << 17, groups=1), UNSUPPORTED, "channels"),
    (dict(groups=5), INVALID, "groups"), (dict(groups=0), INVALID, "groups"), (dict(dtype=0), INVALID, "dtype"),
    (dict(dtype=5), INVALID, "dtype"), (dict(act=3), INVALID, "activation"), (dict(points=1 << 40), UNSUPPORTED, "2^40"),
    (dict(batch=1 << 33, points=1, channels=1, groups=1), UNSUPPORTED, "2^31"),
    (dict(x=ctypes.c_void_p(0x1002)), INVALID, "aligned"), (dict(weight=ODD), INVALID, "aligned"),
    (dict(bias=ODD), INVALID, "aligned"), (dict(stats=ctypes.c_void_p(0x1004)), INVALID, "aligned"),
    (dict(ws=None), WORKSPACE, "workspace"), (dict(ws_bytes=8), WORKSPACE, "workspace"),
    (dict(ws=ctypes.c_void_p(0x1010)), WORKSPACE, "aligned"),
]


@pytest.mark.parametrize("kw,status,word", NORM_BOTH)
def test_norm_rejects_bad_arguments(kw, status, word):
    for call in (_norm_fwd, _norm_bwd):
        assert call(_norm(**kw)) == status
        assert word in _lib.load().ecc_last_error().decode()


def test_norm_rejects_what_one_direction_needs():
    last = _lib.load().ecc_last_error
    for kw, word in ((dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(y=None), "y is"), (dict(y=ODD), "aligned")):
        assert _norm_fwd(_norm(**kw)) == INVALID and word in last().decode()
    assert _norm_bwd(_norm(stats=None)) == INVALID and "stats" in last().decode()
    assert _norm_bwd(_norm(), gy=None) == INVALID and "grad_y" in last().decode()
    assert _norm_bwd(_norm(), gx=None, gw=None, gb=None) == INVALID and "every output" in last().decode()
    for kw in (dict(gx=ODD), dict(gw=ODD), dict(gb=ODD), dict(gy=ODD)):
        assert _norm_bwd(_norm(), **kw) == INVALID and "aligned" in last().decode()
    assert _lib.load().ecc_norm_workspace_bytes(2, 9, 12, 5) == 0
    assert _lib.load().ecc_norm_workspace_bytes(2, 9, 12, 3) > 0


def _xent(**kw):
    a = dict(h=FAKE, w=FAKE, labels=FAKE, rows=4, dim=8, classes=16, dtype=2, ignore=-100, reduction=0, loss=FAKE, stats=FAKE,
             counted=FAKE, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return a


def _xent_fwd(a):
    return _lib.load().ecc_xent_fwd(a["h"], a["w"], a["labels"], a["rows"], a["dim"], a["classes"], a["dtype"], a["ignore"],
                                    a["reduction"], a["loss"], a["stats"], a["counted"], a["ws"], a["ws_bytes"], None)


def _xent_bwd(a, up=FAKE, gh=FAKE, gw=FAKE):
    return _lib.load().ecc_xent_bwd(a["h"], a["w"], a["labels"], a["rows"], a["dim"], a["classes"], a["dtype"], a["ignore"],
                                    a["reduction"], a["stats"], a["counted"], up, gh, gw, a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(h=None), INVALID, "hidden"), (dict(w=None), INVALID, "weight"), (dict(labels=None), INVALID, "labels"),
    (dict(rows=0), INVALID, "rows"), (dict(dim=0), INVALID, "dim"), (dict(classes=0), INVALID, "classes"),
    (dict(rows=1 << 31), UNSUPPORTED, "2^31"), (dict(classes=1 << 31), UNSUPPORTED, "2^31"),
    (dict(dim=1 << 17), UNSUPPORTED, "dim"), (dict(dtype=1), INVALID, "dtype"), (dict(reduction=3), INVALID, "reduction"),
    (dict(h=ctypes.c_void_p(0x1002)), INVALID, "aligned"), (dict(w=ODD), INVALID, "aligned"),
    (dict(labels=ctypes.c_void_p(0x1004)), INVALID, "aligned"), (dict(stats=None), INVALID, "stats"),
    (dict(counted=None), INVALID, "counted"), (dict(stats=ctypes.c_void_p(0x1008)), INVALID, "aligned"),
    (dict(counted=ctypes.c_void_p(0x1004)), INVALID, "aligned"), (dict(ws=None), WORKSPACE, "workspace"),
    (dict(ws_bytes=8), WORKSPACE, "workspace"), (dict(ws=ctypes.c_void_p(0x1010)), WORKSPACE, "aligned"),
])
def test_xent_rejects_bad_arguments(kw, status, word):
    for call in (_xent_fwd, _xent_bwd):
        assert call(_xent(**kw)) == status
        assert word in _lib.load().ecc_last_error().decode()


def test_xent_rejects_what_one_direction_needs():
    last = _lib.load().ecc_last_error
    assert _xent_fwd(_xent(loss=None)) == INVALID and "loss" in last().decode()
    assert _xent_fwd(_xent(loss=ODD)) == INVALID and "aligned" in last().decode()
    assert _xent_bwd(_xent(), up=None) == INVALID and "grad_loss" in last().decode()
    assert _xent_bwd(_xent(), gh=None, gw=None) == INVALID and "every output" in last().decode()
    for kw in (dict(up=ODD), dict(gh=ODD), dict(gw=ODD)):
        assert _xent_bwd(_xent(), **kw) == INVALID and "aligned" in last().decode()
    for back in (0, 1):
        assert _lib.load().ecc_xent_workspace_bytes(0, 8, 16, 2, back) == 0
        assert _lib.load().ecc_xent_workspace_bytes(4, 8, 16, 0, back) == 0
        assert _lib.load().ecc_xent_workspace_bytes(4, 8, 16, 2, back) > 0


def test_layers_refuse_on_the_host():
    x, w = torch.zeros(2, 3, 12), torch.zeros(5, 12)
    for call in (lambda: group_norm_act(x, 3), lambda: linear_cross_entropy(x, w, torch.zeros(2, 3, dtype=torch.int64)),
                 lambda: GroupNormAct(5, 12), lambda: GroupNormAct(0, 12), lambda: GroupNormAct(3, 12, act="tanh"),
                 lambda: LinearCrossEntropy(0, 4), lambda: LinearCrossEntropy(4, 4, reduction="max"),
                 lambda: LinearCrossEntropy(4, 4, dtype=torch.float64)):
        with pytest.raises(ValueError):
            call()
    assert GroupNormAct(3, 12, affine=False).weight is None
    assert LinearCrossEntropy(5, 12, dtype=torch.bfloat16).weight.dtype == torch.bfloat16
