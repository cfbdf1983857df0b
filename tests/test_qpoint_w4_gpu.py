"""The pointwise product with 4-bit letters on the GPU against the fp64 oracle.

Quantisation has one right answer, so the letters and scales are compared bit for bit.  An output is
a sum of exact products taken in fp32 (at most 128 in the tensor cores, then chains of groups) and
rounded once to bf16: within 2^-8 of itself and 2e-5 of the sum of its terms' magnitudes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer

pytestmark = pytest.mark.gpu

ACT = {"none": quan.QUAN_ACT_NONE, "relu": quan.QUAN_ACT_RELU, "silu": quan.QUAN_ACT_SILU}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def bf16(a, shift=0):
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(torch.bfloat16)
    buf = torch.empty(t.numel() + shift, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def letters(Cin, Cout, seed):
    rng = np.random.default_rng(seed)
    mag = np.exp2(rng.integers(-3, 4, size=(4, Cout // 4, 1)))
    return [bf16(rng.normal(size=(Cout // 4, 1, 1, Cin // 4)) * mag[k][:, :, None, None] /
                 np.sqrt(Cin)) for k in range(4)]


def activations(rows, C, seed, shift=0):
    rng = np.random.default_rng(seed)
    return bf16(rng.normal(size=(rows, C)) * np.exp(rng.normal(size=C)) *
                np.exp2(rng.integers(-4, 5, size=(rows, 1))), shift)


def values(w, group):
    return [blocks.w4_letter(f64(v)[:, 0, 0], group)[0] for v in w]


def decode(f):
    """Whole numbers [4, 16 tiles, 64 tiles] and scales [4, 16 tiles, groups] by the documented
    order."""
    L, nt, kt, _ = f.q.shape
    words = f.q.cpu().numpy().view(np.uint32).reshape(L, nt, kt, 8, 4, 4)
    q = np.zeros((L, nt * 16, kt * 64))
    g, t, s = np.meshgrid(np.arange(8), np.arange(4), np.arange(4), indexing="ij")
    for i in range(8):
        n = g + 8 * (i % 2)
        k = 32 * (s // 2) + 8 * t + 4 * (s % 2) + 2 * (i % 4 // 2) + i // 4
        v = ((words >> np.uint32(4 * i)) & np.uint32(15)).astype(np.int64) - 8
        for a in range(nt):
            for b in range(kt):
                q[:, a * 16 + n, b * 64 + k] = v[:, a, b]
    sc = f64(f.scale).reshape(L, nt, -1, 8, 2).transpose(0, 1, 4, 3, 2).reshape(L, nt * 16, -1)
    return q, sc


def check(rows, Cin, Cout, group=64, act="none", vectors=(), seed=0, shift=0):
    w, x = letters(Cin, Cout, seed), activations(rows, Cin, seed + 1, shift)
    f = quan.quantize_w4_weights(*w, group=group)
    z, m = blocks.qpoint(f64(x), values(w, group))
    rng = np.random.default_rng(seed + 2)
    v = {k: torch.from_numpy(rng.uniform(0.5, 1.5, Cout).astype(np.float32)).cuda()
         for k in vectors}
    got = quan.qpointwise_w4(x, f, act=ACT[act], **v)
    if "bias" in v:
        z, m = z + f64(v["bias"]), m + f64(v["bias"])
    if "scale" in v:
        z, m = z * f64(v["scale"]) + f64(v["shift"]), m * f64(v["scale"]) + f64(v["shift"])
    if act == "relu":
        z = np.maximum(z, 0.0)
    elif act == "silu":
        with np.errstate(over="ignore"):
            z = z / (1.0 + np.exp(-z))
    g = f64(got)
    assert np.isfinite(g).all()
    worst = np.max(np.abs(g - z) - (2.0 ** -8 * np.abs(z) + 2e-5 * m))
    assert worst <= 0.0, "past the tolerance by %.3e" % worst
    return x, f, got


@pytest.mark.parametrize("Cin, Cout", [(4, 4), (64, 64), (520, 328), (512, 1024), (36, 2052),
                                       (1100, 516), (252, 60)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_letters(Cin, Cout, group):
    w = letters(Cin, Cout, 3)
    w[2][0, 0, 0, :] = 0.0
    f = quan.quantize_w4_weights(*w, group=group)
    assert (f.Cin, f.Cout, f.group) == (Cin, Cout, group)
    q, s = decode(f)
    n, k = Cout // 4, Cin // 4
    assert not q[:, n:].any() and not q[:, :, k:].any()
    for L in range(4):
        _, wq, ws = blocks.w4_letter(f64(w[L])[:, 0, 0], group)
        assert np.array_equal(s[L, :n], ws) and np.array_equal(q[L, :n, :k], wq)


SHAPES = [(1, 4, 4), (1, 512, 1024), (1, 8192, 512), (1, 4096, 4096), (2, 2048, 260),
          (3, 520, 36), (4, 64, 512), (5, 1024, 1024), (8, 2048, 128), (9, 100, 340),
          (13, 1172, 2804), (16, 512, 512), (17, 36, 2052), (49, 2048, 2048), (64, 1028, 516),
          (65, 256, 64), (200, 300, 20), (1000, 128, 132)]


@pytest.mark.parametrize("rows, Cin, Cout", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_product(rows, Cin, Cout, group):
    check(rows, Cin, Cout, group)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("vectors", [(), ("bias",), ("scale", "shift"),
                                     ("bias", "scale", "shift")])
@pytest.mark.parametrize("rows, Cin, Cout", [(1, 256, 132), (30, 520, 640)])
def test_epilogue(rows, Cin, Cout, vectors, act):
    check(rows, Cin, Cout, act=act, vectors=vectors, seed=11)


@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("rows", [1, 2, 20])
def test_misaligned_input_and_output(rows, shift):
    x, f, got = check(rows, 256, 512, shift=shift, seed=5)
    buf = torch.empty(got.numel() + shift, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:].view(got.shape)
    assert quan.qpointwise_w4(x, f, out=out) is out and torch.equal(out, got)


def test_a_row_does_not_depend_on_the_others():
    # whatever stands beside a pixel in its MMA, infinities and NaN too
    for rows in (2, 7, 30):
        x, f, got = check(rows, 1024, 260, seed=6)
        y = x.clone()
        y[1:, 5] = float("nan")
        y[1:, 700] = float("inf")
        bad = quan.qpointwise_w4(y, f)
        assert torch.equal(bad[0], got[0]) and torch.isnan(bad[1:]).all()


def test_every_product_of_the_hamilton_table():
    w = [bf16(np.full((1, 1, 1, 1), v)) for v in (1.0, 2.0, 4.0, 8.0)]
    f = quan.quantize_w4_weights(*w)
    # max / 7 rounds to bf16 and 7 of it are the value in steps of 7: what the letters stand for
    r, i, j, k = (float(v[0, 0]) for v in values(w, 64))
    assert (2 * r, 2 * i, 2 * j) == (i, j, k) and abs(r - 1.0) < 2.0 ** -8
    y = f64(quan.qpointwise_w4(bf16(np.eye(4)), f))
    block = np.array([[r, -i, -j, -k], [i, r, -k, j], [j, k, r, -i], [k, -j, i, r]])
    assert np.abs(y - block.T).max() <= 2.0 ** -8 * 8 and np.array_equal(np.sign(y), np.sign(block.T))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_infinity_or_nan_in_a_letter(group, bad):
    w = letters(1024, 1024, 1)
    x = activations(3, 1024, 2)
    good = quan.qpointwise_w4(x, quan.quantize_w4_weights(*w, group=group), act=ACT["relu"])
    w[1][130, 0, 0, 5] = bad
    got = quan.qpointwise_w4(x, quan.quantize_w4_weights(*w, group=group), act=ACT["relu"])
    hit = torch.zeros(4, 256, dtype=torch.bool, device="cuda")
    hit[:, 130] = True
    hit = hit.reshape(-1)
    assert torch.isnan(got[:, hit]).all() and torch.equal(got[:, ~hit], good[:, ~hit])


def test_zero_tiny_and_huge_groups():
    w = letters(1024, 64, 7)
    w[0][0] = 0.0
    w[1][3] *= 2.0 ** -125
    w[2][5] *= 2.0 ** 100
    f = quan.quantize_w4_weights(*w, group=32)
    q, s = decode(f)
    for L in range(4):
        _, wq, ws = blocks.w4_letter(f64(w[L])[:, 0, 0], 32)
        assert np.array_equal(s[L, :16], ws) and np.array_equal(q[L, :16], wq)


def test_streams_repeats_leading_shape_and_no_rows():
    for rows, Cin in ((1, 4096), (12, 1024), (60, 512)):
        x, f, got = check(rows, Cin, 512, seed=9)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for stream in (None, s, s.cuda_stream):
            again = quan.qpointwise_w4(x, f, stream=stream)
            s.synchronize()
            torch.cuda.synchronize()
            assert torch.equal(again, got)
    y = quan.qpointwise_w4(x.view(3, 4, 5, 512), f)
    assert y.shape == (3, 4, 5, 512) and torch.equal(y.view(60, 512), got)
    e = torch.empty((0, 4, 512), dtype=torch.bfloat16, device="cuda")
    assert quan.qpointwise_w4(e, f).shape == (0, 4, 512)


def test_captured():
    x, f, got = check(1, 4096, 1024, seed=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = quan.qpointwise_w4(x, f)
    for seed in (1, 2):
        x.copy_(activations(1, 4096, seed))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, quan.qpointwise_w4(x, f))


def test_refuses_on_the_device():
    x, f, _ = check(2, 64, 64)
    with pytest.raises(ValueError, match="x must"):
        quan.qpointwise_w4(x.float(), f)
    with pytest.raises(ValueError, match="x must"):
        quan.qpointwise_w4(x[:, :32], f)
    with pytest.raises(ValueError, match="w.scale"):
        quan.qpointwise_w4(x, f._replace(group=128, Cin=64, scale=f.scale[:2]))
    with pytest.raises(ValueError, match="bias"):
        quan.qpointwise_w4(x, f, bias=torch.zeros(32, device="cuda"))
    with pytest.raises(quan.QuanError):
        quan.qpointwise_w4(x, f, scale=torch.ones(64, device="cuda"))  # no shift
    with pytest.raises(quan.QuanError):
        quan.qpointwise_w4(x, f, out=x)


def test_the_stack_serves_with_4_bit_letters():
    m = Mixer(256, 2, alpha=0.5, seed=1)
    m.quantize_4bit(group=64)
    x = torch.randn(2, 1, 3, 256, device="cuda").to(torch.bfloat16)
    out = m.serve(x)
    rows = lambda t: f64(t).reshape(-1, 256)
    ones = np.ones(256)
    _, n = quan.residual_join(x, pre=m.pre[0], groups=4, eps=m.eps)
    y = x
    for l in range(2):
        h = quan.qpointwise_w4(n, m.w4[l])
        want, mag = blocks.qpoint(rows(n), values(m.letters[l], 64))
        assert (np.abs(rows(h) - want) <= 2.0 ** -8 * np.abs(want) + 2e-5 * mag).all()
        y, n = quan.residual_join(y, h, **m._join(l, x.numel(), False))
    assert torch.equal(out, n)
