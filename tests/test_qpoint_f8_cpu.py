"""The 8-bit pointwise product without a GPU: the oracle's e4m3 and scales against their
definitions, its products against the convolution oracle, and the refusals of the C ABI and the
Python helpers, made before anything is launched."""
import numpy as np
import pytest

import oracle
from oracle import blocks
from paper_2509_05512_gb300 import build, quan

INVALID = quan.QUAN_ERR_INVALID_ARG
UNSUPPORTED = quan.QUAN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return quan.load()


def _e4m3_values():
    """Every non-negative e4m3 value, from its bits: 1 sign, 4 exponent (bias 7), 3 mantissa."""
    out = []
    for b in range(0x7F):  # 0x7f is NaN
        e, m = b >> 3, b & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


def test_round_e4m3():
    v = _e4m3_values()
    assert v.max() == 448.0 and (np.diff(v) > 0).all()
    assert np.array_equal(blocks.round_e4m3(v), v) and np.array_equal(blocks.round_e4m3(-v), -v)
    mid = (v[1:] + v[:-1]) / 2
    even = np.where(np.arange(len(mid)) % 2 == 0, v[:-1], v[1:])  # ties to the even pattern
    assert np.array_equal(blocks.round_e4m3(mid), even)
    for step in (1e-9, -1e-9):
        want = v[1:] if step > 0 else v[:-1]
        assert np.array_equal(blocks.round_e4m3(mid * (1 + step)), want)


def test_round_e4m3_agrees_with_torch():
    torch = pytest.importorskip("torch")
    a = np.random.default_rng(0).uniform(-448, 448, 20000)
    a = np.concatenate([a, a * 1e-3, a * 1e-5]).astype(np.float32)
    want = torch.from_numpy(a).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(blocks.round_e4m3(a), want)


def test_f8_scale():
    a = np.array([0.0, 448.0, 448.0001, 224.0, 1.0, 1.75, 1.7500001, 1e-45, 3e38, np.inf, np.nan])
    s = blocks.f8_scale(a)
    assert s[0] == 1.0 and s[1] == 1.0 and s[2] == 2.0 and s[3] == 0.5
    assert s[4] == 2.0 ** -8 and s[5] == 2.0 ** -8 and s[6] == 2.0 ** -7
    assert s[7] == 2.0 ** -126 and np.isnan(s[9:]).all()
    assert (a[1:7] / s[1:7] <= 448).all() and (a[1:7] / s[1:7] > 223.9).all()


def test_oracle_product_matches_the_convolution_oracle():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(1, 3, 2, 20))
    w = [rng.normal(size=(7, 1, 1, 5)) for _ in range(4)]
    got, mag = blocks.qpoint(x.reshape(6, 20), [v[:, 0, 0] for v in w])
    want = oracle.qconv2d(x, *w, stride=1, pad=0)
    assert np.allclose(got.reshape(want.shape), want, atol=1e-12) and (mag >= np.abs(got)).all()
    dy = rng.normal(size=want.shape)
    got, _ = blocks.qpoint(dy.reshape(6, 28), [v[:, 0, 0] for v in w], transpose=True)
    want = oracle.qconv2d_bwd_data(dy, *w, H=3, W=2, stride=1, pad=0)
    assert np.allclose(got.reshape(want.shape), want, atol=1e-12)


A = {k: 0x10000000 * (i + 1) for i, k in enumerate(
    ["x", "wq", "ws", "bias", "scale", "shift", "work", "out", "wr", "wi", "wj", "wk", "q"])}


def _fwd(lib, **kw):
    a = dict(A, rows=8, Cin=64, Cout=128, act=1, bytes=1 << 26)
    a.update(kw)
    return lib.quan_qpoint_f8_fwd(a["x"], a["wq"], a["ws"], a["bias"], a["scale"], a["shift"],
                                  a["rows"], a["Cin"], a["Cout"], a["act"], a["work"],
                                  a["bytes"], a["out"], None)


def _bwd(lib, **kw):
    a = dict(A, rows=8, Cin=64, Cout=128, bytes=1 << 26)
    a.update(kw)
    return lib.quan_qpoint_f8_bwd_data(a["x"], a["wq"], a["ws"], a["rows"], a["Cin"], a["Cout"],
                                       a["work"], a["bytes"], a["out"], None)


COMMON = [dict(x=None), dict(wq=None), dict(ws=None), dict(out=None), dict(rows=-1), dict(Cin=6),
          dict(Cout=0), dict(Cout=10), dict(x=A["x"] + 1), dict(wq=A["wq"] + 8),
          dict(ws=A["ws"] + 2), dict(out=A["x"]), dict(out=A["wq"] + 64), dict(out=A["ws"])]


@pytest.mark.parametrize("bad", COMMON + [
    dict(act=3), dict(scale=None), dict(shift=None), dict(bias=A["bias"] + 1),
    dict(out=A["shift"]),
])
def test_product_refuses(lib, bad):
    assert _fwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


@pytest.mark.parametrize("bad", COMMON)
def test_gradient_refuses(lib, bad):
    assert _bwd(lib, **bad) == INVALID


def test_product_limits(lib):
    assert _fwd(lib, rows=0) == quan.QUAN_OK
    assert _fwd(lib, rows=1 << 31) == UNSUPPORTED
    assert _fwd(lib, Cin=1 << 21) == UNSUPPORTED and _fwd(lib, Cout=1 << 21) == UNSUPPORTED
    assert _bwd(lib, rows=1 << 30, Cin=4, Cout=1 << 12) == UNSUPPORTED
    assert lib.quan_qpoint_f8_workspace_size(8, 6, 4) == 0
    need = lib.quan_qpoint_f8_workspace_size(4096, 512, 512)
    if need:
        assert _fwd(lib, rows=4096, Cin=512, Cout=512, work=None, bytes=0) == INVALID
        assert _fwd(lib, rows=4096, Cin=512, Cout=512, bytes=need - 1) == INVALID
        assert _fwd(lib, rows=4096, Cin=512, Cout=512, work=A["work"] + 16) == INVALID
        assert _fwd(lib, rows=4096, Cin=512, Cout=512, work=A["x"]) == INVALID


def test_weights_refuse(lib):
    def call(**kw):
        a = dict(A, Cin=64, Cout=128, t=0)
        a.update(kw)
        return lib.quan_f8_weights(a["wr"], a["wi"], a["wj"], a["wk"], a["Cin"], a["Cout"],
                                   a["t"], a["q"], a["ws"], None)
    for bad in (dict(wr=None), dict(wk=None), dict(q=None), dict(ws=None), dict(Cin=2),
                dict(Cout=0), dict(q=A["q"] + 8), dict(wi=A["wi"] + 1), dict(q=A["wj"]),
                dict(ws=A["q"])):
        assert call(**bad) == INVALID, bad
    assert lib.quan_f8_weights_bytes(20, 28, 0) == 4 * 7 * 16
    assert lib.quan_f8_weights_bytes(20, 28, 1) == 4 * 5 * 16
    assert lib.quan_f8_weights_bytes(20, 27, 0) == 0


def test_helpers_refuse():
    torch = pytest.importorskip("torch")
    w = [torch.zeros(4, 1, 1, 8, dtype=torch.bfloat16) for _ in range(4)]
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.quantize_f8_weights(*w)
    with pytest.raises(ValueError, match="pointwise"):
        quan.quantize_f8_weights(*[torch.zeros(4, 3, 3, 8) for _ in range(4)])
    f = quan.F8Weights(None, None, 32, 16, False)
    x = torch.zeros(2, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="forward letters"):
        quan.qpointwise_f8_backward_data(x, f)
    with pytest.raises(ValueError, match="transposed letters"):
        quan.qpointwise_f8(x, f._replace(transposed=True))
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.qpointwise_f8(x, f)
