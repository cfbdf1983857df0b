"""The join whose norm comes out in 8 bits without a GPU: sizes, and the refusals of the C ABI and
the Python helpers, made before anything is launched."""
import pytest

from paper_2509_05512_gb300 import build, quan

INVALID = quan.QUAN_ERR_INVALID_ARG
UNSUPPORTED = quan.QUAN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return quan.load()


A = {k: 0x10000000 * (i + 1) for i, k in enumerate(
    ["x", "h", "y", "n", "q", "scale", "post", "gate", "pre", "wq", "ws", "out", "bias", "s", "t"])}


def test_sizes(lib):
    assert lib.quan_f8_rows_bytes(3, 340) == 3 * 4 * 96 and lib.quan_f8_rows_scales(3, 340) == 512
    assert lib.quan_f8_rows_bytes(129, 1028) == 129 * 4 * 272
    assert lib.quan_f8_rows_scales(129, 1028) == 4 * 3 * 256
    for rows, C in ((0, 64), (-1, 64), (4, 0), (4, 66)):
        assert lib.quan_f8_rows_bytes(rows, C) == 0 and lib.quan_f8_rows_scales(rows, C) == 0


def _join(lib, **kw):
    a = dict(A, rows=8, C=64, groups=4, images=2, dtype=0, alpha=1.0, eps=1e-5, p=0.1, seed=1,
             offset=0, counter=None)
    a.update(kw)
    return lib.quan_residual_join_f8_fwd(
        a["x"], a["h"], a["post"], a["gate"], a["pre"], a["rows"], a["C"], a["groups"],
        a["images"], a["dtype"], a["alpha"], a["eps"], a["p"], a["seed"], a["offset"],
        a["counter"], a["y"], a["n"], a["q"], a["scale"], None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=9), dict(images=0), dict(C=0), dict(C=66), dict(C=66, groups=1),
    dict(groups=2), dict(dtype=5), dict(alpha=float("inf")), dict(eps=0.0), dict(p=2.0),
    dict(post=A["post"] + 2), dict(h=A["h"] + 1), dict(h=None), dict(x=None), dict(y=None),
    dict(q=None), dict(scale=None), dict(pre=None), dict(h=None, y=None),
    dict(h=None, y=None, post=None), dict(q=A["q"] + 8), dict(scale=A["scale"] + 2),
    dict(n=A["n"] + 1), dict(y=A["x"] + 64), dict(n=A["x"]), dict(y=A["h"]), dict(n=A["y"]),
    dict(q=A["x"]), dict(q=A["h"]), dict(q=A["n"] + 16), dict(scale=A["q"]), dict(scale=A["gate"]),
    dict(n=A["h"], dtype=1),  # bf16 over fp32
])
def test_join_refuses(lib, bad):
    assert _join(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_join_limits(lib):
    assert _join(lib, rows=0) == quan.QUAN_OK
    assert _join(lib, C=8196) == UNSUPPORTED and _join(lib, C=8196, groups=1) == UNSUPPORTED
    assert _join(lib, rows=1 << 31) == UNSUPPORTED


def _read(lib, **kw):
    a = dict(A, rows=8, C=64)
    a.update(kw)
    return lib.quan_f8_rows_dequant(a["q"], a["scale"], a["rows"], a["C"], a["out"], None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(C=0), dict(C=6), dict(q=None), dict(scale=None), dict(out=None),
    dict(q=A["q"] + 8), dict(scale=A["scale"] + 1), dict(out=A["out"] + 1), dict(out=A["q"] + 16),
    dict(out=A["scale"] + 64)])
def test_reading_back_refuses(lib, bad):
    assert _read(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_reading_back_limits(lib):
    assert _read(lib, rows=0) == quan.QUAN_OK
    assert _read(lib, rows=1 << 31) == UNSUPPORTED and _read(lib, C=1 << 21) == UNSUPPORTED


def _product(lib, **kw):
    a = dict(A, rows=8, Cin=64, Cout=128, act=1)
    a.update(kw)
    return lib.quan_qpoint_f8_rows_fwd(a["q"], a["scale"], a["wq"], a["ws"], a["bias"], a["s"],
                                       a["t"], a["rows"], a["Cin"], a["Cout"], a["act"], a["out"],
                                       None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(scale=None), dict(wq=None), dict(ws=None), dict(out=None), dict(rows=-1),
    dict(Cin=6), dict(Cout=0), dict(q=A["q"] + 8), dict(scale=A["scale"] + 2), dict(act=3),
    dict(s=None), dict(out=A["q"]), dict(out=A["scale"] + 128), dict(out=A["wq"])])
def test_product_refuses(lib, bad):
    assert _product(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_product_limits(lib):
    assert _product(lib, rows=0) == quan.QUAN_OK
    assert _product(lib, rows=1 << 31) == UNSUPPORTED
    assert _product(lib, Cin=1 << 21) == UNSUPPORTED


def test_helpers_refuse():
    torch = pytest.importorskip("torch")
    x, v = torch.zeros(2, 8), torch.ones(8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.residual_join_f8(x, pre=v)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        quan.residual_join_f8(x.half(), pre=v)
    with pytest.raises(TypeError):
        quan.residual_join_f8(x)
    rows = quan.F8Rows(torch.zeros(2, 4, 16, dtype=torch.float8_e4m3fn), torch.zeros(4, 1, 128), 8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.dequantize_f8_rows(rows)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.qpointwise_f8(rows, quan.F8Weights(None, None, 8, 16, False))
