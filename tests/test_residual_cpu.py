"""Dropout and the residual join without a GPU: the oracle's generator against published known
answers and its gradients against differences, and the refusals of the C ABI and the Python
helpers, made before anything is launched."""
import numpy as np
import pytest

from oracle import blocks
from paper_2509_05512_gb300 import build, quan

INVALID = quan.QUAN_ERR_INVALID_ARG
UNSUPPORTED = quan.QUAN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return quan.load()


def test_philox_known_answer():
    # the generator's published vectors for an all-zero counter and key, and key bits alone
    assert [hex(v) for v in blocks.philox4x32([0], 0)[0]] == \
        ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    assert not np.array_equal(blocks.philox4x32([0], 1 << 32), blocks.philox4x32([0], 1))


def test_dropout_factor_limits():
    assert np.array_equal(blocks.dropout_factor(9, 0.0, 1), np.ones(9))
    assert np.array_equal(blocks.dropout_factor(9, 1.0, 1), np.zeros(9))
    f = blocks.dropout_factor(80000, 0.25, 12345, 7)
    # 80000 draws: the share kept is within six standard deviations
    assert abs((f > 0).mean() - 0.75) < 6 * np.sqrt(0.25 * 0.75 / 80000)
    assert set(np.unique(f)) == {0.0, 65536.0 / 49152.0}


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("images", [None, 1, 3])
@pytest.mark.parametrize("norms", ["both", "post", "pre", "none"])
def test_oracle_gradient_against_differences(groups, images, norms):
    rng = np.random.default_rng(groups + 10 * (images or 0))
    rows, C, eps = 6, 12, 1e-3
    x, h = rng.normal(size=(2, rows, C))
    post = rng.uniform(0.5, 1.5, C) if norms in ("both", "post") else None
    pre = rng.uniform(0.5, 1.5, C) if norms in ("both", "pre") else None
    gate = None if images is None else rng.uniform(0.2, 1.0, (images, C))
    factor = blocks.dropout_factor(rows * C, 0.25, 5).reshape(rows, C)
    dy, dn = rng.normal(size=(2, rows, C))
    kw = dict(alpha=0.7, groups=groups, eps=eps, factor=factor)
    y, _ = blocks.join(x, h, post, gate, pre, **kw)
    grads = blocks.join_backward(dy, dn if pre is not None else None, y, h, post, gate, pre, **kw)

    def loss(x, h, post, gate, pre):
        y, n = blocks.join(x, h, post, gate, pre, **kw)
        return (dy * y).sum() + (0.0 if n is None else (dn * n).sum())

    args = [x, h, post, gate, pre]
    for k, g in enumerate(grads):
        if args[k] is None:
            assert g is None
            continue
        d = rng.normal(size=args[k].shape)
        t = 1e-5  # central difference: error t^2 f''' / 6, rounding 1e-16 / t
        up = loss(*[a + t * d if i == k else a for i, a in enumerate(args)])
        down = loss(*[a - t * d if i == k else a for i, a in enumerate(args)])
        assert abs((up - down) / (2 * t) - (g * d).sum()) < 1e-6 * max(1.0, abs((g * d).sum()))


FAKE = 0x10000  # never dereferenced: every case below fails validation first


def _dropout(lib, x=FAKE, n=64, dtype=0, p=0.5, seed=1, offset=0, counter=None, out=0x900000):
    return lib.quan_dropout(x, n, dtype, p, seed, offset, counter, out, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(out=None), dict(n=-1), dict(dtype=2), dict(p=-0.1), dict(p=1.5),
    dict(p=float("nan")), dict(counter=4), dict(x=FAKE + 1), dict(out=FAKE + 2),
    dict(out=0x900002, dtype=1), dict(counter=0x900008),
])
def test_dropout_refuses(lib, bad):
    assert _dropout(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_dropout_empty_and_too_large(lib):
    assert _dropout(lib, x=None, out=None, n=0) == quan.QUAN_OK
    assert _dropout(lib, n=1 << 41) == UNSUPPORTED


A = {k: 0x10000000 * (i + 1) for i, k in enumerate(
    ["x", "h", "y", "n", "dy", "dn", "dx", "dh", "post", "gate", "pre", "dpost", "dgate",
     "dpre", "ws"])}


def _fwd(lib, **kw):
    a = dict(A, rows=8, C=64, groups=4, images=2, dtype=0, alpha=1.0, eps=1e-5, p=0.1, seed=1,
             offset=0, counter=None)
    a.update(kw)
    return lib.quan_residual_join_fwd(
        a["x"], a["h"], a["post"], a["gate"], a["pre"], a["rows"], a["C"], a["groups"],
        a["images"], a["dtype"], a["alpha"], a["eps"], a["p"], a["seed"], a["offset"],
        a["counter"], a["y"], a["n"], None)


def _bwd(lib, **kw):
    a = dict(A, rows=8, C=64, groups=4, images=2, dtype=0, alpha=1.0, eps=1e-5, p=0.1, seed=1,
             offset=0, counter=None, bytes=1 << 20)
    a.update(kw)
    return lib.quan_residual_join_bwd(
        a["dy"], a["dn"], a["y"], a["h"], a["post"], a["gate"], a["pre"], a["rows"], a["C"],
        a["groups"], a["images"], a["dtype"], a["alpha"], a["eps"], a["p"], a["seed"],
        a["offset"], a["counter"], a["ws"], a["bytes"], a["dx"], a["dh"], a["dpost"],
        a["dgate"], a["dpre"], None)


COMMON = [
    dict(rows=-1), dict(rows=9), dict(images=0), dict(C=0), dict(C=66), dict(groups=2),
    dict(dtype=5), dict(alpha=float("inf")), dict(eps=0.0), dict(eps=float("nan")), dict(p=2.0),
    dict(post=A["post"] + 2), dict(h=A["h"] + 1), dict(h=None),
]


@pytest.mark.parametrize("bad", COMMON + [
    dict(x=None), dict(y=None), dict(n=None), dict(pre=None),
    dict(h=None, y=None), dict(h=None, y=None, post=None),        # gate without a branch
    dict(y=A["x"] + 64), dict(n=A["x"]), dict(y=A["h"]), dict(n=A["y"]), dict(y=A["gate"]),
])
def test_join_refuses(lib, bad):
    assert _fwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


@pytest.mark.parametrize("bad", COMMON + [
    dict(dn=None), dict(y=None), dict(pre=None), dict(dpre=None), dict(dpost=None),
    dict(dgate=None), dict(dh=None), dict(dx=None), dict(dpost=A["dpost"] + 2),
    dict(dy=None, dn=None, y=None, pre=None, dpre=None),
])
def test_join_backward_refuses(lib, bad):
    assert _bwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_join_limits(lib):
    assert _fwd(lib, C=8196) == UNSUPPORTED
    assert _fwd(lib, C=16384, groups=1) == UNSUPPORTED
    assert _fwd(lib, rows=1 << 39) == UNSUPPORTED
    assert _fwd(lib, rows=0) == quan.QUAN_OK
    for bad in (dict(rows=9), dict(groups=3), dict(C=6)):
        a = dict(dict(rows=8, C=64, groups=4, images=2), **bad)
        assert lib.quan_residual_join_bwd_workspace_size(a["rows"], a["C"], a["groups"],
                                                         a["images"]) == 0


def test_helpers_refuse_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.dropout(x, 0.5, 1)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        quan.dropout(x.half(), 0.5, 1)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.residual_join(x, x)
    with pytest.raises(ValueError, match="dy or dn"):
        quan.residual_join_backward(None, None, None)
