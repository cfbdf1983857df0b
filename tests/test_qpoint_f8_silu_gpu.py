"""SiLU of the 8-bit pointwise product over its whole range, on both kernels (CUDA cores for few
rows, tensor cores for many), against z / (1 + e^-z) in 64 bits.

Each input row is one magnitude times an identity letter, so that a pre-activation is one exact
product and the tolerance can be taken of the result itself: one bf16 rounding (2^-8), the exponential of
an argument of at most 128 with fp32's relative error (2^-15) and, below z = -87.3, where the
divisor passes 2^126 and its reciprocal counts as 0, 88.8 e^-87.3 < 2^-119."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu

Z = [-0.25, -1.0, -8.0, -20.0, -40.0, -44.0, -48.0, -60.0, -80.0, -88.0, -96.0, -112.0, -1e4,
     -2.0 ** 50, -1e20, -1e30, -2.0 ** 100, -1.75 * 2.0 ** 126, 0.0, 1.0, 20.0, 88.0, 1e30]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield
    assert quan.quan_device_status()[0] == quan.QUAN_OK


def silu(z):
    return np.where(z < -700.0, -0.0, z / (1.0 + np.exp(-np.maximum(z, -700.0))))


def identity(Q):
    r = torch.eye(Q).reshape(Q, 1, 1, Q).to(torch.bfloat16).cuda()
    return quan.quantize_f8_weights(r, *(torch.zeros_like(r) for _ in range(3)))


@pytest.mark.parametrize("Q", [16, 64, 136])
@pytest.mark.parametrize("rows", [1, 3, 300])
def test_silu_range(rows, Q):
    f = identity(Q)
    for first in range(0, len(Z), rows):
        z = np.resize(Z[first:first + rows], rows)
        a = np.repeat(z[:, None], 4 * Q, axis=1)
        a[:, 1::3] *= 0.25  # a neighbour of another size
        x = torch.from_numpy(a).to(torch.bfloat16).cuda()
        got = quan.qpointwise_f8(x, f, act=quan.QUAN_ACT_SILU).double().cpu().numpy()
        want = silu(blocks.f8_rows(x.double().cpu().numpy()))
        assert np.isfinite(got).all()
        tol = (2.0 ** -8 + 2.0 ** -15) * np.abs(want) + 2.0 ** -119
        worst = np.abs(got - want) - tol
        at = np.unravel_index(np.argmax(worst), worst.shape)
        assert worst.max() <= 0.0, "z %g: %g, not %g" % (a[at], got[at], want[at])


@pytest.mark.parametrize("rows", [1, 3, 300])
def test_silu_of_shifted_and_infinite_sums(rows):
    # the vectors take z far down, and past fp32: -inf / (1 + inf) is NaN, as by the formula
    Q = 32
    x = torch.ones(rows, 4 * Q, dtype=torch.bfloat16, device="cuda")
    scale = torch.ones(4 * Q, device="cuda")
    shift = torch.zeros(4 * Q, device="cuda")
    shift[1], shift[2], shift[3] = -1e6, -1e20, -1e36
    scale[4], scale[5] = -3e38, 3e38
    shift[4], shift[5] = -3e38, 3e38
    got = quan.qpointwise_f8(x, identity(Q), scale=scale, shift=shift,
                             act=quan.QUAN_ACT_SILU).double().cpu().numpy()
    assert (np.abs(got[:, 1:4]) <= 2.0 ** -119).all()
    assert np.isnan(got[:, 4]).all() and (got[:, 5] == np.inf).all()
    one = silu(np.array(1.0))
    assert (np.abs(got[:, [0] + list(range(6, 4 * Q))] - one) <= 2.0 ** -8 * one).all()
