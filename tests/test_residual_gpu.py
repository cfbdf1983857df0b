"""Dropout and the residual join on the GPU against the fp64 oracle.

Tolerances, from the arithmetic: a bf16 result is an fp32 value rounded once, so within 2^-8 of
it; the fp32 values in front of that carry sums of at most 8192 terms, taken as chains of at most
16 per thread and a tree of 10 levels, an approximate reciprocal square root (2^-22) and a dozen
roundings: below 1e-5 of the row's largest term.  Column sums are chains of at most a few hundred
terms, then trees: below 2e-5 of the sum of the terms' magnitudes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def dev(a, dtype, shift=0):
    """A tensor of `dtype` whose first element lies `shift` elements into its storage."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(dtype)
    buf = torch.empty(t.numel() + shift, dtype=dtype, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def close(got, want, scale, dtype, what):
    """|got - want| <= the rounding to dtype and 1e-5 of `scale` (a row's largest term)."""
    got = f64(got).reshape(want.shape)
    assert np.isfinite(got).all(), what
    tol = 1e-5 * scale + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
    worst = np.max(np.abs(got - want) - tol) if want.size else 0.0
    assert worst <= 0.0, "%s: past the tolerance by %.3e" % (what, worst)


def row_scale(*parts):
    s = sum(np.abs(p) for p in parts)
    return s.max(axis=1, keepdims=True)


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, shift", [(1, 0), (7, 0), (8, 0), (9, 3), (4099, 0), (4096, 1),
                                      (1 << 20, 0), (12345677, 0)])
def test_dropout_values(dtype, n, shift):
    x = dev(np.random.default_rng(n).normal(size=n), DT[dtype], shift)
    seed, offset = 0x9E3779B97F4A7C15, (1 << 32) - 3  # counters past 32 bits
    got = quan.dropout(x, 0.3, seed, offset)
    f = blocks.dropout_factor(n, 0.3, seed, offset)
    want = torch.from_numpy(f64(x).astype(np.float32) * f.astype(np.float32)).to(DT[dtype])
    assert torch.equal(got.cpu(), want)  # one product in fp32, one rounding: the same bits


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -16, 1.0 - 2.0 ** -16])
def test_dropout_extreme_p(p):
    x = dev(np.random.default_rng(0).normal(size=70001), torch.float32)
    f = blocks.dropout_factor(x.numel(), p, 3)
    want = torch.from_numpy(f64(x).astype(np.float32) * f.astype(np.float32))
    assert torch.equal(quan.dropout(x, p, 3).cpu(), want)


def test_dropout_drops_infinities_and_nan():
    f = blocks.dropout_factor(64, 0.5, 11)
    a = np.where(np.arange(64) % 2 == 0, np.inf, np.nan)
    got = f64(quan.dropout(dev(a, torch.float32), 0.5, 11))
    assert np.array_equal(got == 0.0, f == 0.0)
    assert np.array_equal(np.isnan(got), np.isnan(a) & (f > 0))


def test_dropout_in_place_other_stream_and_empty():
    x = dev(np.random.default_rng(1).normal(size=5000), torch.bfloat16)
    want = quan.dropout(x, 0.5, 9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = quan.dropout(x, 0.5, 9, stream=s)
    b = quan.dropout(x, 0.5, 9, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
    assert quan.dropout(x, 0.5, 9, out=x) is x
    assert torch.equal(x, want)
    e = torch.empty((0, 8), dtype=torch.float32, device="cuda")
    assert quan.dropout(e, 0.5, 1).shape == (0, 8)


def test_dropout_counter_moves_the_mask_of_a_captured_graph():
    x = torch.ones(4096, device="cuda")
    counter = torch.zeros((), dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        quan.dropout(x, 0.5, 5, 100, counter=counter, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        quan.dropout(x, 0.5, 5, 100, counter=counter, out=out)
    for step in (0, 512, 1 << 33):
        counter.fill_(step)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(f64(out), blocks.dropout_factor(4096, 0.5, 5, 100 + step))


# ------------------------------------------------------------------ the join

def make(shape, dtype, seed, gate="channel", norms="both", shift=0, names=("x", "h", "dy", "dn")):
    rng = np.random.default_rng(seed)
    C, N = shape[-1], shape[0]
    d = {k: dev(rng.normal(size=shape) * (2.0 if k == "h" else 1.0), DT[dtype], shift)
         for k in names}
    vec = lambda *s: torch.from_numpy(rng.uniform(0.3, 1.5, s).astype(np.float32)).cuda()
    kw = {"post": vec(C) if norms in ("both", "post") else None,
          "pre": vec(C) if norms in ("both", "pre") else None,
          "gate": {"none": None, "channel": vec(C), "image": vec(N, C)}[gate]}
    return d, kw


def oracle_args(d, kw, C, p, seed, offset, groups, alpha, eps):
    rows = {k: f64(t).reshape(-1, C) for k, t in d.items()}
    n = rows["x"].size
    f = None if p == 0.0 else blocks.dropout_factor(n, p, seed, offset).reshape(-1, C)
    return rows, {k: f64(v) for k, v in kw.items()}, dict(alpha=alpha, groups=groups, eps=eps,
                                                          factor=f)


def check_both(shape, dtype, *, groups=1, gate="channel", norms="both", p=0.0, alpha=1.0,
               shift=0, eps=1e-5, seed=1):
    C = shape[-1]
    d, kw = make(shape, dtype, seed, gate, norms, shift)
    rng = dict(p=p, seed=77, offset=13)
    common = dict(kw, alpha=alpha, groups=groups, eps=eps, **rng)
    rows, vec, okw = oracle_args(d, kw, C, p, 77, 13, groups, alpha, eps)
    y, n = quan.residual_join(d["x"], d["h"], **common)
    wy, wn = blocks.join(rows["x"], rows["h"], **vec, **okw)
    close(y, wy, row_scale(rows["x"], wy - rows["x"]), dtype, "y")
    if kw["pre"] is None:
        assert n is None
    else:
        # an error of y moves n by n / y of it: at most the row's largest n / y times it
        close(n, wn, row_scale(wn), dtype, "n")
    # the gradients read the y that was written
    yr = f64(y).reshape(-1, C)
    dn = d["dn"] if kw["pre"] is not None else None
    got = quan.residual_join_backward(d["dy"], dn, y, d["h"], **common)
    want = blocks.join_backward(rows["dy"], rows["dn"] if dn is not None else None, yr,
                                rows["h"], **vec, **okw)
    # the terms that dx and dh are differences of: dy and dn pre / rms(y); s gate post / rms(h)
    rms = lambda v: np.sqrt((v.reshape(len(v), groups, -1) ** 2).mean(axis=2, keepdims=True) +
                            eps).repeat(C // groups, axis=2).reshape(v.shape)
    tx = row_scale(rows["dy"])
    if dn is not None:
        tx = tx + row_scale(rows["dn"] * vec["pre"] / rms(yr))
    close(got[0], want[0], tx, dtype, "dx")
    s = abs(alpha) * tx * (1.0 if okw["factor"] is None else okw["factor"])
    s = s * blocks._gate_rows(vec["gate"], len(yr), C)
    if vec["post"] is not None:
        s = s * vec["post"] / rms(rows["h"])
    close(got[1], want[1], row_scale(s), dtype, "dh")
    # magnitudes of the terms of the column sums, dx standing for the terms it is a difference of
    f = 1.0 if okw["factor"] is None else okw["factor"]
    at = dict(alpha=abs(alpha), groups=groups, eps=eps, factor=np.broadcast_to(f, yr.shape))
    absw = blocks.join_backward(np.broadcast_to(tx, yr.shape), None, None, np.abs(rows["h"]),
                                vec["post"], vec["gate"], None, **at)
    mag = [absw[2], absw[3], None if dn is None else np.abs(rows["dn"] * yr / rms(yr)).sum(axis=0)]
    for name, g, w, m in zip(("dpost", "dgate", "dpre"), got[2:], want[2:], mag):
        assert (g is None) == (w is None), name
        if g is not None:
            assert g.dtype == torch.float32 and tuple(g.shape) == w.shape
            assert (np.abs(f64(g) - w) <= 2e-5 * m + 1e-30).all(), name
    return d, common, y, n, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("shape", [
    (1, 1, 1, 4), (1, 1, 1, 512), (2, 3, 5, 8), (3, 7, 7, 64), (2, 5, 3, 340), (1, 9, 9, 100),
    (2, 4, 4, 1028), (1, 3, 3, 2048), (1, 1, 5, 4100), (1, 1, 3, 8192), (4, 33, 31, 32),
])
def test_join(shape, groups, dtype):
    check_both(shape, dtype, groups=groups, p=0.25, alpha=0.5)


@pytest.mark.parametrize("norms", ["both", "post", "pre", "none"])
@pytest.mark.parametrize("gate", ["none", "channel", "image"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_join_forms(dtype, gate, norms):
    check_both((3, 5, 7, 96), dtype, gate=gate, norms=norms, groups=4, p=0.1, alpha=-1.5)
    check_both((3, 5, 7, 96), dtype, gate=gate, norms=norms, groups=1)


@pytest.mark.parametrize("shape", [(64, 7, 7, 128), (300, 2, 2, 64), (700, 1, 1, 260),
                                   (5, 61, 59, 64), (2, 112, 112, 16)])
def test_join_images(shape):
    # few and many images, fewer rows an image than a block holds side by side, many blocks
    check_both(shape, "bf16", gate="image", groups=4, p=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_join_alignment(dtype, shift):
    check_both((2, 3, 5, 64), dtype, groups=4, p=0.25, shift=shift)


def test_join_gradient_against_differences():
    # fp32 tensors; the loss in fp64 from the oracle's forward, its slope along random directions
    # from a central difference of step 1e-5 (error below 1e-6), the kernel's from its gradients:
    # they agree within the gradients' own tolerance summed over the elements
    shape, C, groups, eps = (3, 4, 5, 48), 48, 4, 1e-3
    d, kw = make(shape, "f32", 5, "image")
    common = dict(kw, alpha=0.8, groups=groups, eps=eps, p=0.25, seed=77, offset=13)
    rows, vec, okw = oracle_args(d, kw, C, 0.25, 77, 13, groups, 0.8, eps)
    y, _ = quan.residual_join(d["x"], d["h"], **common)
    got = quan.residual_join_backward(d["dy"], d["dn"], y, d["h"], **common)
    args = [rows["x"], rows["h"], vec["post"], vec["gate"], vec["pre"]]
    rng = np.random.default_rng(6)

    def loss(a):
        wy, wn = blocks.join(*a, **okw)
        return (rows["dy"] * wy).sum() + (rows["dn"] * wn).sum()

    for k, g in enumerate(got):
        v = rng.normal(size=args[k].shape)
        t = 1e-5
        slope = (loss([a + t * v if i == k else a for i, a in enumerate(args)]) -
                 loss([a - t * v if i == k else a for i, a in enumerate(args)])) / (2 * t)
        terms = f64(g).reshape(v.shape) * v
        assert abs(terms.sum() - slope) <= 2e-5 * np.abs(terms).sum() + 1e-5


def test_join_special_rows():
    # a row of zeros, a dropped infinity without a post-norm, a NaN that stays in its row
    C = 64
    x = torch.zeros(4, C, device="cuda")
    h = torch.zeros(4, C, device="cuda")
    one = torch.ones(C, device="cuda")
    y, n = quan.residual_join(x, h, post=one, pre=one)
    assert not y.any() and not n.any()
    f = blocks.dropout_factor(4 * C, 0.5, 3).reshape(4, C)
    h[1, int(np.argmin(f[1]))] = float("inf")
    h[2, int(np.argmax(f[2]))] = float("nan")
    y, n = quan.residual_join(x, h, pre=one, p=0.5, seed=3)
    assert not y[[0, 1, 3]].any() and not n[[0, 1, 3]].any()
    assert int(torch.isnan(y).sum()) == 1 and bool(torch.isnan(n[2]).all())
    # and has no part in a gradient
    g = torch.randn(4, C, device="cuda")
    dx, dh, _, dgate, _ = quan.residual_join_backward(g, None, None, h[:2].repeat(2, 1),
                                                      gate=one, p=0.5, seed=3)
    keep = torch.from_numpy(f > 0).cuda()
    assert not dh[~keep].any() and bool(torch.isfinite(dh).all())
    # everything dropped: the branch has no part, and no gradient
    h = torch.randn(4, C, device="cuda")
    x = torch.randn(4, C, device="cuda")
    y, n = quan.residual_join(x, h, post=one, pre=one, p=1.0)
    assert torch.equal(y, x)
    dx, dh, dpost, _, _ = quan.residual_join_backward(x, h, y, h, post=one, pre=one, p=1.0)
    assert not dh.any() and not dpost.any() and bool(torch.isfinite(dx).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_alone(dtype):
    x = dev(np.random.default_rng(2).normal(size=(3, 5, 5, 320)), DT[dtype])
    dn = dev(np.random.default_rng(3).normal(size=(3, 5, 5, 320)), DT[dtype])
    pre = torch.rand(320, device="cuda") + 0.5
    y, n = quan.residual_join(x, pre=pre, groups=4)
    assert y is None
    rows, w = f64(x).reshape(-1, 320), f64(pre)
    want = blocks.join(rows, pre=w, groups=4)[1]
    close(n, want, row_scale(want), dtype, "n")
    dx, dh, dpost, dgate, dpre = quan.residual_join_backward(None, dn, x, pre=pre, groups=4)
    assert dh is None and dpost is None and dgate is None
    wdx, _, _, _, wdpre = blocks.join_backward(None, f64(dn).reshape(-1, 320), rows, pre=w,
                                               groups=4)
    close(dx, wdx, row_scale(wdx), dtype, "dx")
    assert np.abs(f64(dpre) - wdpre).max() <= 2e-5 * np.abs(f64(dn)).sum(axis=(0, 1, 2)).max() * 4


def test_join_without_rows():
    x = torch.empty((0, 3, 3, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    y, n = quan.residual_join(x, x, post=w, gate=w, pre=w)
    assert y.shape == x.shape and n.shape == x.shape
    _, _, dpost, dgate, dpre = quan.residual_join_backward(x, x, x, x, post=w, gate=w, pre=w)
    for g in (dpost, dgate, dpre):
        assert g.shape == (64,) and not g.any()


def test_join_in_place_streams_and_repeats():
    shape = (4, 13, 11, 256)
    d, common, y, n, got = check_both(shape, "bf16", groups=4, gate="image", p=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s, s.cuda_stream):
        again = quan.residual_join(d["x"], d["h"], stream=stream, **common)
        grads = quan.residual_join_backward(d["dy"], d["dn"], y, d["h"], stream=stream, **common)
        s.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(again + grads, (y, n) + got):
            assert torch.equal(a, b)  # fixed order of every sum: the same bits
    dy, h = d["dy"].clone(), d["h"].clone()
    grads = quan.residual_join_backward(dy, d["dn"], y, h, dx=dy, dh=h, **common)
    for a, b in zip(grads, got):
        assert torch.equal(a, b)
    x, h = d["x"].clone(), d["h"].clone()
    quan.residual_join(x, h, y=x, n=h, **common)
    assert torch.equal(x, y) and torch.equal(h, n)


def test_join_refuses_on_the_device():
    x = torch.zeros(4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    with pytest.raises(ValueError, match="gate"):
        quan.residual_join(x, x.clone(), gate=torch.ones(3, 64, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        quan.residual_join(torch.zeros(64, 64, device="cuda").t()[:4], x)
    with pytest.raises(ValueError, match="h must"):
        quan.residual_join(x, x.bfloat16())
    with pytest.raises(quan.QuanError):
        quan.residual_join(x, x.clone(), pre=w, eps=0.0)
    with pytest.raises(quan.QuanError):
        quan.residual_join(x, x, y=x)  # y may be x, but not h
    with pytest.raises(ValueError, match="counter"):
        quan.dropout(x, 0.5, 1, counter=torch.zeros(1, device="cuda"))
