"""The gradient that distillation sends through the mixing stack's last norm, against 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.distill import distill
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer, distillation

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_the_gain_s_gradient_is_the_formula_s(seed, T):
    # n = pre u, u = y / rms(y): dL/dpre = sum over pixels of dn u.  The kernels' logits are n in bf16, of a
    # y that was not rounded yet: each off by at most 3 2^-8 of itself (n, y and y's part in the rms, half a
    # step each), so that q is off by the factor e^(2 delta), delta = 3 2^-8 max |n| / T, and dn is rounded
    # once more.  fp32 sums and powers stay below 1e-5 of the terms' magnitudes.
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = Mixer(64, 1, seed=5)
    x = torch.randn(1, 6, 6, 64, generator=g, device="cuda").to(torch.bfloat16)
    index = torch.randint(0, 64, (1, 6, 6, 4), generator=g, device="cuda")
    teacher = torch.randn(1, 6, 6, 4, generator=g, device="cuda")
    _, dn = distillation(m, x, index, teacher, temperature=T, training=False)
    got = m.backward(dn)["pre"][1].double().cpu().numpy()
    rows = lambda t: t.detach().double().cpu().numpy().reshape(36, -1)
    y = rows(m.y[1]).reshape(36, 4, 16)
    u = (y / np.sqrt((y ** 2).mean(axis=2, keepdims=True) + m.eps)).reshape(36, 64)
    w, slots = np.full(36, 1.0 / 36), (index.cpu().numpy().reshape(36, 4), rows(teacher))
    pre = m.pre[1].double().cpu().numpy()
    _, _, dz, q, share = distill(u * pre, *slots, w, T)
    delta = 3 * 2.0 ** -8 * np.abs(u * pre).max(axis=1, keepdims=True) / T
    off = 2.0 ** -8 * np.abs(dz) + 1.01 * T / 36 * q * np.expm1(2 * delta)
    tol = (np.abs(u) * (off + 1e-5 * T / 36 * (q + share))).sum(axis=0)
    assert (np.abs(got - (dz * u).sum(axis=0)) <= tol).all()
    # and the formula's is the loss's, by differences in 64 bits: the second is off by h^2 / 6 of the third
    # derivative, of the order of E |d u|^3 < 1e3, and by the loss's rounding over h
    d = np.random.default_rng(seed).normal(size=64)
    loss = lambda s: w @ distill(u * (pre + s * d), *slots, w, T)[0]
    h = 1e-4
    assert abs((loss(h) - loss(-h)) / (2 * h) - ((dz * u).sum(axis=0) * d).sum()) <= 1e-5
