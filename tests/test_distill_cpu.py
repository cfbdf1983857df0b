"""The distillation loss without a GPU: the oracle's gradient against central differences and its
loss against the definition's limits, and the refusals of the C ABI and the Python helpers, made
before anything is launched."""
import numpy as np
import pytest

from oracle.distill import distill
from paper_2509_05512_gb300 import build, quan

INVALID = quan.QUAN_ERR_INVALID_ARG
UNSUPPORTED = quan.QUAN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return quan.load()


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_oracle_gradient_is_the_loss_differences(T):
    rng = np.random.default_rng(0)
    z = rng.normal(size=(4, 9))
    index = rng.integers(0, 9, size=(4, 5))
    index[1, 2] = -1
    index[2] = 9
    index[3] = 4  # five slots of one class
    t, g = rng.normal(size=(4, 5)), rng.normal(size=4)
    dz = distill(z, index, t, g, T)[2]
    assert not dz[2].any() and distill(z, index, t, g, T)[0][2] == 0.0
    d, h = rng.normal(size=z.shape), 1e-5  # error h^2 f''' / 6, rounding 1e-16 / h
    up, down = (g @ distill(z + s * h * d, index, t, g, T)[0] for s in (1, -1))
    assert abs((up - down) / (2 * h) - (dz * d).sum()) < 1e-8


def test_oracle_loss_of_the_teacher_itself_is_zero():
    rng = np.random.default_rng(1)
    z = rng.normal(size=(3, 6))
    index = np.tile(np.arange(6), (3, 1))
    loss, _, dz, q, share = distill(z, index, z, np.ones(3), 2.0)
    assert np.allclose(loss, 0, atol=1e-14) and np.allclose(dz, 0, atol=1e-14)
    assert np.allclose(q, share) and np.allclose(q.sum(1), 1)


A = {k: 0x10000000 * (i + 1) for i, k in enumerate(
    ["z", "index", "teacher", "dloss", "loss", "lse", "dz"])}
BASE = dict(A, rows=8, classes=100, pitch=104, top=10, dtype=0, tdtype=1, bits=64, T=1.0, scale=1.0)


def _sizes(a):
    return (a["rows"], a["classes"], a["pitch"], a["top"], a["dtype"], a["tdtype"], a["bits"],
            a["T"])


def _fwd(lib, **kw):
    a = dict(BASE, **kw)
    return lib.quan_distill_fwd(a["z"], a["index"], a["teacher"], *_sizes(a), a["loss"], a["lse"],
                                None)


def _bwd(lib, **kw):
    a = dict(BASE, **kw)
    return lib.quan_distill_bwd(a["dloss"], a["z"], a["lse"], a["index"], a["teacher"], *_sizes(a),
                                a["scale"], a["dz"], None)


def _both(lib, **kw):
    a = dict(BASE, **kw)
    return lib.quan_distill_fwd_bwd(a["z"], a["index"], a["teacher"], a["dloss"], *_sizes(a),
                                    a["scale"], a["loss"], a["dz"], None)


COMMON = [
    dict(z=None), dict(index=None), dict(teacher=None), dict(rows=-1), dict(classes=0),
    dict(pitch=99), dict(top=0), dict(dtype=2), dict(tdtype=-1), dict(bits=16), dict(T=0.0),
    dict(T=float("nan")), dict(T=1e7), dict(T=1e-7), dict(z=A["z"] + 1), dict(index=A["index"] + 4),
    dict(teacher=A["teacher"] + 2),
]
NAN = float("nan")


@pytest.mark.parametrize("bad", COMMON + [
    dict(loss=None), dict(lse=None), dict(loss=A["z"]), dict(lse=A["loss"] + 4),
    dict(loss=A["loss"] + 2), dict(lse=A["index"]), dict(loss=A["teacher"] + 4)])
def test_loss_refuses(lib, bad):
    assert _fwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


@pytest.mark.parametrize("bad", COMMON + [
    dict(lse=None), dict(dz=None), dict(dz=A["z"] + 4), dict(dz=A["dz"] + 1), dict(dz=A["lse"]),
    dict(dz=A["dloss"]), dict(dz=A["teacher"]), dict(dz=A["index"] + 64), dict(dloss=A["dloss"] + 1),
    dict(scale=NAN), dict(scale=float("inf"))])
def test_gradient_refuses(lib, bad):
    assert _bwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


@pytest.mark.parametrize("bad", COMMON + [
    dict(loss=None), dict(dz=None), dict(loss=A["dz"]), dict(dz=A["z"] + 4), dict(loss=A["dloss"]),
    dict(scale=NAN)])
def test_both_refuse(lib, bad):
    assert _both(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


@pytest.mark.parametrize("call", [_fwd, _bwd, _both])
def test_limits(lib, call):
    assert call(lib, rows=0) == quan.QUAN_OK
    assert call(lib, top=257) == UNSUPPORTED
    assert call(lib, rows=1 << 31) == UNSUPPORTED
    assert call(lib, classes=1 << 24, pitch=1 << 24) == UNSUPPORTED
    assert call(lib, rows=1 << 30, pitch=1 << 12) == UNSUPPORTED


def test_helpers_refuse():
    torch = pytest.importorskip("torch")
    z, i, t = torch.zeros(2, 8), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3)
    calls = (lambda *a: quan.distill_loss(*a), lambda *a: quan.distill_loss_and_gradient(*a),
             lambda *a: quan.distill_loss_backward(None, a[0], torch.zeros(2), *a[1:]))
    for call in calls:
        with pytest.raises(ValueError, match="CUDA tensor"):
            call(z, i, t)
        with pytest.raises(ValueError, match="bfloat16 or float32"):
            call(z.half(), i, t)


def test_no_load_through_the_read_only_path():
    # the grid starts while the one before it may still write its inputs (the logits, lse), and such
    # a load may be moved in front of its wait
    import os
    import re
    path = os.path.join(os.path.dirname(build.LIB_PATH), "csrc", "distill.cu")
    with open(path) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert not re.search(r"__ldg\b|ld\.global\.nc|const\s+\w+\s*\*\s*__restrict__", text)
