"""The pointwise product with 4-bit letters without a GPU: the oracle's quantisation against its
definition, sizes, and the refusals of the C ABI and the Python helpers."""
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


def test_oracle_quantisation():
    w = np.zeros((3, 70))
    w[0, :5] = [7.0, -3.4, 2.5, 3.5, -7.0]
    w[1, 64:] = 2.0 ** -140
    w[2, 3], w[2, 69] = np.inf, 1.0
    v, q, s = blocks.w4_letter(w, 64)
    assert s.shape == (3, 2) and s[0, 0] == 1.0 and s[0, 1] == 1.0
    assert list(q[0, :5]) == [7, -3, 2, 4, -7] and list(v[0, :5]) == [7, -3, 2, 4, -7]
    assert s[1, 1] == 1.0 and not q[1].any()  # max / 7 is nothing in bf16
    assert np.isnan(s[2, 0]) and np.isnan(v[2, :64]).all() and s[2, 1] == 0.142578125
    assert q[2, 69] == 7
    rng = np.random.default_rng(0)
    w = rng.normal(size=(20, 200))
    v, q, s = blocks.w4_letter(w, 32)
    each = np.repeat(s, 32, 1)[:, :200]
    # half a step, and 7 steps fall short of the maximum by the scale's rounding
    assert (np.abs(v - w) <= each * (0.5 + 7 * 2.0 ** -8)).all()


def test_sizes(lib):
    assert lib.quan_w4_weights_bytes(512, 1024) == 4 * 16 * 2 * 512
    assert lib.quan_w4_weights_bytes(20, 28) == 4 * 512
    assert lib.quan_w4_weights_scales(520, 68, 32) == 4 * 2 * 5 * 16
    assert lib.quan_w4_weights_scales(520, 68, 128) == 4 * 2 * 2 * 16
    assert lib.quan_w4_weights_bytes(6, 4) == 0 and lib.quan_w4_weights_scales(64, 64, 48) == 0


A = {k: 0x10000000 * (i + 1) for i, k in enumerate(
    ["x", "wq", "ws", "bias", "scale", "shift", "out", "wr", "wi", "wj", "wk", "q"])}


def _fwd(lib, **kw):
    a = dict(A, rows=8, Cin=64, Cout=128, group=64, act=1)
    a.update(kw)
    return lib.quan_qpoint_w4_fwd(a["x"], a["wq"], a["ws"], a["bias"], a["scale"], a["shift"],
                                  a["rows"], a["Cin"], a["Cout"], a["group"], a["act"], a["out"],
                                  None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(wq=None), dict(ws=None), dict(out=None), dict(rows=-1), dict(Cin=6),
    dict(Cout=0), dict(Cout=10), dict(group=16), dict(group=0), dict(x=A["x"] + 1),
    dict(wq=A["wq"] + 8), dict(ws=A["ws"] + 2), dict(out=A["x"]), dict(out=A["wq"] + 64),
    dict(out=A["ws"]), dict(act=3), dict(scale=None), dict(shift=None), dict(bias=A["bias"] + 1),
    dict(out=A["shift"])])
def test_product_refuses(lib, bad):
    assert _fwd(lib, **bad) == INVALID
    assert lib.quan_last_error_message()


def test_product_limits(lib):
    assert _fwd(lib, rows=0) == quan.QUAN_OK
    assert _fwd(lib, rows=(1 << 20) + 1) == UNSUPPORTED
    assert _fwd(lib, Cin=1 << 21) == UNSUPPORTED and _fwd(lib, Cout=1 << 21) == UNSUPPORTED


def test_weights_refuse(lib):
    def call(**kw):
        a = dict(A, Cin=64, Cout=128, group=64)
        a.update(kw)
        return lib.quan_w4_weights(a["wr"], a["wi"], a["wj"], a["wk"], a["Cin"], a["Cout"],
                                   a["group"], a["q"], a["ws"], None)
    for bad in (dict(wr=None), dict(wk=None), dict(q=None), dict(ws=None), dict(Cin=2),
                dict(Cout=0), dict(group=96), dict(q=A["q"] + 8), dict(wi=A["wi"] + 1),
                dict(q=A["wj"]), dict(ws=A["q"])):
        assert call(**bad) == INVALID, bad
    assert call(Cin=1 << 21) == UNSUPPORTED


def test_helpers_refuse():
    torch = pytest.importorskip("torch")
    w = [torch.zeros(4, 1, 1, 8, dtype=torch.bfloat16) for _ in range(4)]
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.quantize_w4_weights(*w)
    with pytest.raises(ValueError, match="pointwise"):
        quan.quantize_w4_weights(*[torch.zeros(4, 3, 3, 8) for _ in range(4)])
    with pytest.raises(ValueError, match="group"):
        quan.quantize_w4_weights(*w, group=48)
    with pytest.raises(ValueError, match="CUDA tensor"):
        quan.qpointwise_w4(torch.zeros(2, 32, dtype=torch.bfloat16),
                           quan.W4Weights(None, None, 32, 16, 64))


def test_no_load_through_the_read_only_path():
    # the grid starts while the one before it may still write its inputs, and such a load may be
    # moved in front of its wait
    import os
    import re
    path = os.path.join(os.path.dirname(build.LIB_PATH), "csrc", "qpoint_w4.cu")
    with open(path) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert not re.search(r"__ldg\b|ld\.global\.nc|const\s+\w+\s*\*\s*__restrict__", text)
