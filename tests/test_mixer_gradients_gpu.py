"""The mixing stack's backward pass, every step of it against the fp64 oracle: each join's, product's
and weight gradient's results, from what the step before it wrote, with parameters of their own in
every block.  So a gradient that goes to the wrong block, is left out, or is taken of other letters
shows.

Tolerances: a bf16 result is within 2^-8 of itself and 1e-5 (joins) or 2e-5 (products) of the
terms it is a sum of, for its fp32 sums and roundings; an fp32 sum over pixels within 2e-5 of its
terms' magnitudes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield
    assert quan.quan_device_status()[0] == quan.QUAN_OK


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def rows(t):
    return None if t is None else f64(t).reshape(-1, t.shape[-1])


def within(got, want, tol, what):
    got = f64(got).reshape(want.shape)
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - want) - tol).max()
    assert worst <= 0.0, "%s: past the tolerance by %.3e" % (what, worst)


def rms(v, groups, eps):
    r = np.sqrt((v.reshape(len(v), groups, -1) ** 2).mean(axis=2, keepdims=True) + eps)
    return r.repeat(v.shape[1] // groups, axis=2).reshape(v.shape)


def widest(a):
    return np.abs(a).max(axis=1, keepdims=True)


def check_join(got, dy, dn, y, h, post, gate, pre, what, *, groups, eps, alpha, factor):
    want = blocks.join_backward(dy, dn, y, h, post, gate, pre, groups=groups, eps=eps, alpha=alpha,
                                factor=factor)
    terms = widest(dn * pre / rms(y, groups, eps)) + (0.0 if dy is None else widest(dy))
    within(got[0], want[0], 2.0 ** -8 * np.abs(want[0]) + 1e-5 * terms, what + " dx")
    mag = np.abs(dn * y / rms(y, groups, eps)).sum(axis=0)
    within(got[4], want[4], 2e-5 * mag, what + " dpre")
    if h is None:
        return
    s = abs(alpha) * terms * factor
    back = widest(s * gate * post / rms(h, groups, eps))
    within(got[1], want[1], 2.0 ** -8 * np.abs(want[1]) + 1e-5 * back, what + " dh")
    normed = np.abs(h) / rms(h, groups, eps)
    within(got[2], want[2], 2e-5 * (s * gate * normed).sum(axis=0), what + " dpost")
    within(got[3], want[3], 2e-5 * (s * normed * post).sum(axis=0), what + " dgate")


def letter_gradients(x, dy):
    """(values, magnitudes) of dL/dW for the four letters of x W, from rows of x and dL/d(x W)."""
    xs, ds = np.split(x, 4, axis=1), np.split(dy, 4, axis=1)
    value, mag = [0.0] * 4, [0.0] * 4
    for co in range(4):
        for ci in range(4):
            value[co ^ ci] = value[co ^ ci] + blocks._SIGN[co, ci] * (ds[co].T @ xs[ci])
            mag[co ^ ci] = mag[co ^ ci] + np.abs(ds[co]).T @ np.abs(xs[ci])
    return value, mag


@pytest.mark.parametrize("C, groups, p, training", [(96, 4, 0.25, True), (256, 1, 0.5, True),
                                                    (64, 4, 0.25, False)])
def test_every_gradient(monkeypatch, C, groups, p, training):
    depth, N, H, alpha, eps = 3, 3, 9, 0.5, 1e-5
    m = Mixer(C, depth, groups=groups, p=p, alpha=alpha, eps=eps, seed=7)
    m.counter.fill_(1000)
    g = torch.Generator(device="cuda").manual_seed(C)
    for name in ("pre", "post", "gate"):
        for v in getattr(m, name):
            v.copy_(0.5 + torch.rand(C, generator=g, device="cuda"))
    x = torch.randn(N, H, H, C, generator=g, device="cuda").to(torch.bfloat16)
    dn = torch.randn(N, H, H, C, generator=g, device="cuda").to(torch.bfloat16)

    joins, products = [], []

    def record(name, into):
        call = getattr(quan, name)

        def wrapped(*a, **k):
            into.append(call(*a, **k))
            return into[-1]
        monkeypatch.setattr(quan, name, wrapped)

    m.forward(x, training=training)
    record("residual_join_backward", joins)
    record("qpointwise_f8_backward_data", products)
    grads = m.backward(dn)
    assert len(joins) == depth + 1 and len(products) == depth

    per = -(-x.numel() // 8)
    vec = {name: [f64(v) for v in getattr(m, name)] for name in ("pre", "post", "gate")}
    dy, dn_rows = None, rows(dn)
    for step, l in enumerate(reversed(range(depth))):
        factor = blocks.dropout_factor(x.numel(), p if training else 0.0, 7, 1000 + l * per) \
            .reshape(-1, C)
        got = joins[step]
        check_join(got, dy, dn_rows, rows(m.y[l + 1]), rows(m.h[l]), vec["post"][l],
                   vec["gate"][l], vec["pre"][l + 1], "block %d" % l, groups=groups, eps=eps,
                   alpha=alpha, factor=factor)
        assert grads["post"][l] is got[2] and grads["gate"][l] is got[3]
        assert grads["pre"][l + 1] is got[4]
        dy, dh = rows(got[0]), rows(got[1])
        value, mag = letter_gradients(rows(m.n[l]), dh)
        for L in range(4):
            assert grads["letters"][l][L].dtype == torch.float32
            within(grads["letters"][l][L], value[L], 2e-5 * mag[L], "letter %d of %d" % (L, l))
        letters = [blocks.f8_letter(f64(w)[:, 0, 0])[0] for w in m.letters[l]]
        want, mag = blocks.qpoint(blocks.f8_rows(dh), letters, transpose=True)
        within(products[step], want, 2.0 ** -8 * np.abs(want) + 2e-5 * mag, "dn %d" % l)
        dn_rows = rows(products[step])
    check_join(joins[depth], dy, dn_rows, rows(m.y[0]), None, None, None, vec["pre"][0], "input",
               groups=groups, eps=eps, alpha=1.0, factor=None)
    assert grads["dx"] is joins[depth][0] and grads["pre"][0] is joins[depth][4]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("groups", [1, 4])
def test_norm_alone_by_channel(dtype, groups):
    # each channel's sum against its own terms
    g = torch.Generator(device="cuda").manual_seed(groups)
    x, dn = (torch.randn(3, 17, 5, 320, generator=g, device="cuda").to(dtype) for _ in range(2))
    dn = dn * torch.logspace(-3, 3, 320, device="cuda").to(dtype)
    pre = torch.rand(320, generator=g, device="cuda") + 0.5
    dpre = quan.residual_join_backward(None, dn, x, pre=pre, groups=groups)[4]
    want = rows(dn) * rows(x) / rms(rows(x), groups, 1e-5)
    within(dpre, want.sum(axis=0), 2e-5 * np.abs(want).sum(axis=0), "dpre")
