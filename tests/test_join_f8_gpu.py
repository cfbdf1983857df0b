"""The residual join whose norm comes out in 8 bits on the GPU.

Quantisation has one right answer: the rows read back are compared bit for bit with the oracle's
quantisation of the bf16 norm that the same call keeps.  That norm is held to the oracle's join as
residual_join's is (an fp32 value below 1e-5 of the row's largest term away, rounded once to bf16:
2^-8); with a statistic for each component the call gives residual_join's own bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def dev(a, dtype, shift=0):
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(dtype)
    buf = torch.empty(t.numel() + shift, dtype=dtype, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def make(shape, dtype, seed, gate="channel", post=True, shift=0):
    rng = np.random.default_rng(seed)
    C, N = shape[-1], shape[0]
    vec = lambda *s: torch.from_numpy(rng.uniform(0.3, 1.5, s).astype(np.float32)).cuda()
    x = dev(rng.normal(size=shape) * np.exp(rng.normal(size=C)), DT[dtype], shift)
    h = dev(2.0 * rng.normal(size=shape), DT[dtype], shift)
    kw = {"post": vec(C) if post else None, "pre": vec(C),
          "gate": {"none": None, "channel": vec(C), "image": vec(N, C)}[gate]}
    return x, h, kw


def quantised(n):
    """What bf16 rows stand for in 8 bits, by the oracle."""
    return blocks.f8_rows(f64(n).reshape(-1, n.shape[-1])).reshape(n.shape)


def same(a, b):
    a, b = f64(a), np.asarray(b)
    assert np.array_equal(np.isnan(a), np.isnan(b))
    ok = ~np.isnan(a)
    assert np.array_equal(a[ok], b[ok])


def check(shape, dtype="bf16", groups=4, gate="channel", alpha=0.5, p=0.0, post=True, seed=0,
          shift=0, branch=True):
    x, h, kw = make(shape, dtype, seed, gate, post, shift)
    if not branch:
        h, kw = None, {"pre": kw["pre"]}
    args = dict(kw, alpha=alpha, groups=groups, p=p, seed=5, offset=100)
    y, n, n8 = quan.residual_join_f8(x, h, keep=True, **args)
    back = quan.dequantize_f8_rows(n8)
    assert back.shape == x.shape and back.dtype == torch.bfloat16
    same(back, quantised(n))
    y1, n1 = quan.residual_join(x, h, **args)
    if groups == 4:
        assert y1 is None and y is None or torch.equal(y, y1)
        if dtype == "bf16":
            assert torch.equal(n, n1)
        else:
            assert torch.equal(n, n1.to(torch.bfloat16))
    C = shape[-1]
    f = None if p == 0.0 else blocks.dropout_factor(x.numel(), p, 5, 100).reshape(-1, C)
    o = {k: f64(v) for k, v in kw.items()}
    wy, wn = blocks.join(f64(x).reshape(-1, C), None if h is None else f64(h).reshape(-1, C),
                         alpha=alpha, groups=groups, factor=f, **o)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for got, want, rounding in ((y, wy, half), (n, wn, 2.0 ** -8)):
        if got is None:
            continue
        got = f64(got).reshape(want.shape)
        tol = rounding * np.abs(want) + 1e-5 * np.abs(want).max(axis=1, keepdims=True)
        assert (np.abs(got - want) <= tol).all()
    # without n in bf16: the same rows
    y2, none, m8 = quan.residual_join_f8(x, h, **args)
    assert none is None and (y is None or torch.equal(y2, y))
    assert torch.equal(m8.q.view(torch.uint8), n8.q.view(torch.uint8))
    rows = x.numel() // C
    assert torch.equal(m8.scale[:, :, :rows], n8.scale[:, :, :rows])
    # its padding is zero
    assert not f64(n8.q.float())[..., C // 4:].any()
    return x, h, args, y, n, n8


SHAPES = [(1, 1, 1, 4), (1, 1, 1, 512), (3, 5, 2, 64), (2, 7, 3, 100), (5, 31, 29, 340),
          (2, 3, 3, 516), (4, 9, 9, 256), (1, 13, 11, 1024), (3, 5, 1, 2048), (2, 3, 5, 4096),
          (1, 2, 3, 8192), (2, 2, 2, 8180), (1, 5, 5, 4100), (40, 3, 3, 36), (2, 150, 1, 132)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values(shape, groups, dtype):
    check(shape, dtype, groups)


@pytest.mark.parametrize("shape", [(3, 4, 5, 64), (2, 3, 3, 340), (2, 3, 1, 4096)])
@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("kw", [dict(gate="image"), dict(gate="none"), dict(post=False),
                                dict(p=0.3), dict(p=0.3, gate="image", dtype="f32"),
                                dict(branch=False), dict(branch=False, dtype="f32")])
def test_variants(shape, groups, kw):
    check(shape, groups=groups, seed=1, **kw)


@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_misaligned_tensors(shift, dtype):
    x, h, args, y, n, n8 = check((3, 5, 7, 256), dtype, shift=shift, seed=2)
    out = dev(np.zeros(x.shape), torch.bfloat16, shift)
    assert quan.dequantize_f8_rows(n8, out=out) is out
    assert torch.equal(out, quan.dequantize_f8_rows(n8))
    y2, n2, m8 = quan.residual_join_f8(x, h, n=out, **args)
    assert n2 is out and torch.equal(out, n)


def test_in_place_given_outputs_streams_and_no_rows():
    x, h, args, y, n, n8 = check((3, 8, 8, 128), seed=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        y2, n2, m8 = quan.residual_join_f8(x, h, keep=True, stream=stream, **args)
        back = quan.dequantize_f8_rows(m8, stream=stream)
        s.synchronize()
        assert torch.equal(y2, y) and torch.equal(n2, n)
        assert torch.equal(back, quan.dequantize_f8_rows(n8))
    into = quan.F8Rows(torch.zeros_like(n8.q.view(torch.uint8)).view(n8.q.dtype),
                       torch.zeros_like(n8.scale), 128)
    a, b = x.clone(), h.clone()
    y2, n2, m8 = quan.residual_join_f8(a, b, y=a, n=b, n8=into, **args)
    assert y2 is a and n2 is b and m8 is into
    assert torch.equal(a, y) and torch.equal(b, n)
    assert torch.equal(into.q.view(torch.uint8), n8.q.view(torch.uint8))
    rows = x.numel() // 128
    assert torch.equal(into.scale[:, :, :rows], n8.scale[:, :, :rows])
    assert not into.scale[:, :, rows:].any()  # what stands behind the rows is left as it was
    e = x[:0]
    y0, n0, e8 = quan.residual_join_f8(e, e, keep=True, **args)
    assert y0.shape == e.shape and quan.dequantize_f8_rows(e8).shape == e.shape


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("C", [64, 340, 2048])
def test_zeros_and_what_is_not_finite(groups, C):
    x, _, kw = make((1, 9, 1, C), "bf16", 4)
    x[0, 1] = 0.0
    x[0, 2, 0, 0] = float("inf")
    x[0, 3, 0, C // 4] = float("nan")
    x[0, 4] *= 2.0 ** -100
    x[0, 5] *= 2.0 ** 60
    _, n, n8 = quan.residual_join_f8(x, pre=kw["pre"], groups=groups, keep=True)
    same(quan.dequantize_f8_rows(n8), quantised(n))
    assert not n[0, 1].any() and (n8.scale[:, :, 1] == 1).all()
    assert torch.isnan(n8.scale[:, :, 2]).any() and torch.isnan(n8.scale[:, :, 3]).any()
    w = quan.quantize_f8_weights(*[torch.randn(16, 1, 1, C // 4, device="cuda").to(torch.bfloat16)
                                   for _ in range(4)])
    a, b = quan.qpointwise_f8(n8, w), quan.qpointwise_f8(n, w)
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.isnan(a[0, 2:4]).all()
    keep = [0, 1, 4, 5, 6, 7, 8]
    assert torch.equal(a[:, keep], b[:, keep])


PRODUCTS = [((1, 1, 1, 512), 1024), ((1, 1, 3, 520), 36), ((1, 4, 4, 1024), 512),
            ((2, 10, 15, 512), 512), ((1, 16, 8, 340), 260), ((3, 17, 19, 1100), 64),
            ((1, 1, 1, 4), 4), ((5, 40, 50, 256), 128)]


@pytest.mark.parametrize("shape, Cout", PRODUCTS)
def test_product_of_the_rows_has_the_bits_of_the_bf16_product(shape, Cout):
    x, _, kw = make(shape, "bf16", 6)
    _, n, n8 = quan.residual_join_f8(x, pre=kw["pre"], groups=4, keep=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = quan.quantize_f8_weights(*[torch.randn(Cout // 4, 1, 1, shape[-1] // 4, generator=g,
                                               device="cuda").to(torch.bfloat16)
                                   for _ in range(4)])
    v = [torch.rand(Cout, generator=g, device="cuda") for _ in range(3)]
    for args in (dict(), dict(bias=v[0], scale=v[1], shift=v[2], act=quan.QUAN_ACT_SILU)):
        want = quan.qpointwise_f8(n, w, **args)
        got = quan.qpointwise_f8(n8, w, **args)
        assert got.shape == want.shape and torch.equal(got, want)
        out = torch.empty_like(want)
        assert quan.qpointwise_f8(n8, w, out=out, **args) is out and torch.equal(out, want)


def test_captured_with_a_counter():
    x, h, kw = make((2, 8, 8, 256), "bf16", 7)
    counter = torch.zeros((), dtype=torch.int64, device="cuda")
    args = dict(kw, groups=4, p=0.5, seed=9, counter=counter)
    w = quan.quantize_f8_weights(*[torch.randn(64, 1, 1, 64, device="cuda").to(torch.bfloat16)
                                   for _ in range(4)])
    quan.qpointwise_f8(quan.residual_join_f8(x, h, **args)[2], w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        y, n, n8 = quan.residual_join_f8(x, h, keep=True, **args)
        back = quan.dequantize_f8_rows(n8)
        out = quan.qpointwise_f8(n8, w)
    for step in (0, 7):
        counter.fill_(step)
        g.replay()
        torch.cuda.synchronize()
        y1, n1 = quan.residual_join(x, h, **args)
        assert torch.equal(y, y1) and torch.equal(n, n1)
        same(back, quantised(n1))
        assert torch.equal(out, quan.qpointwise_f8(n1, w))


def test_past_two_to_the_31_elements():
    rows, C = 540000, 4096  # 2.2e9 channels: 4.4 GB, 2.2 GB in 8 bits
    x = torch.randn(rows, 64, device="cuda").to(torch.bfloat16).repeat(1, C // 64)
    pre = torch.rand(C, device="cuda") + 0.5
    _, _, n8 = quan.residual_join_f8(x, pre=pre, groups=1)
    at = torch.tensor([0, 1, 131072, 262143, 524287, 524288, rows - 1], device="cuda")
    back = quan.dequantize_f8_rows(n8)[at]
    _, n, m8 = quan.residual_join_f8(x[at].clone(), pre=pre, groups=1, keep=True)
    assert torch.equal(back, quan.dequantize_f8_rows(m8))
    same(back, quantised(n))


@pytest.mark.parametrize("groups", [1, 4])
def test_the_stack_keeps_its_results(groups):
    # the stack's forward pass by the calls it is made of: a join in bf16, which the product quantises
    m = Mixer(96, 3, groups=groups, p=0.25, alpha=0.5, seed=3)
    x = torch.randn(2, 9, 9, 96, device="cuda").to(torch.bfloat16)
    out = m.forward(x)
    _, n = quan.residual_join(x, pre=m.pre[0], groups=groups, eps=m.eps)
    y = x
    for l in range(m.depth):
        assert torch.equal(m.n[l], n)
        h = quan.qpointwise_f8(n, m.w[l])
        y, n = quan.residual_join(y, h, **m._join(l, x.numel(), True))
        assert torch.equal(m.h[l], h) and torch.equal(m.y[l + 1], y)
    assert torch.equal(out, n)


def test_refuses_on_the_device():
    x, h, args, y, n, n8 = check((2, 3, 3, 64), seed=8)
    with pytest.raises(ValueError, match="h must"):
        quan.residual_join_f8(x, h.float(), **args)
    with pytest.raises(ValueError, match="n must"):
        quan.residual_join_f8(x, h, n=n.float(), **args)
    with pytest.raises(ValueError, match="n8"):
        quan.residual_join_f8(x, h, n8=n8._replace(channels=60), **args)
    with pytest.raises(ValueError, match="n8"):
        quan.residual_join_f8(x[:1], h[:1], n8=n8, **args)
    with pytest.raises(ValueError, match="multiple of 4"):
        quan.residual_join_f8(x.view(-1, 6), pre=torch.ones(6, device="cuda"))
    with pytest.raises(ValueError, match="x.scale"):
        quan.dequantize_f8_rows(n8._replace(scale=n8.scale[:, :, :64]))
    with pytest.raises(ValueError, match="x.q"):
        quan.dequantize_f8_rows(n8._replace(q=n8.q.view(torch.uint8)))
    w = quan.quantize_f8_weights(*[torch.zeros(4, 1, 1, 8, device="cuda", dtype=torch.bfloat16)
                                   for _ in range(4)])
    with pytest.raises(ValueError, match="channels"):
        quan.qpointwise_f8(n8, w)
    with pytest.raises(quan.QuanError):
        quan.residual_join_f8(x, h, n=x, **args)


@pytest.mark.parametrize("C", [4, 20, 28, 32, 36, 60, 68, 244, 508, 512, 516, 524, 1028, 2060, 8188])
@pytest.mark.parametrize("rows", [1, 2, 7, 33, 1000])
def test_rows_of_any_width_read_back(C, rows):
    # any bytes and scales (powers of two, so that a value is exact in bf16), padding that is not 0, a
    # block without a scale: every element with its own block's scale, wherever components begin
    Q, pitch, blocks = C // 4, (C + 63) // 64 * 16, (C + 511) // 512
    g = torch.Generator(device="cuda").manual_seed(C + rows)
    q = torch.randint(0, 127, (rows, 4, pitch), generator=g, device="cuda", dtype=torch.uint8)
    q += 128 * torch.randint(0, 2, q.shape, generator=g, device="cuda", dtype=torch.uint8)
    scale = torch.randint(-20, 20, (4, blocks, (rows + 127) // 128 * 128), generator=g, device="cuda")
    scale = torch.exp2(scale.float())
    scale[2, blocks - 1, rows - 1] = float("nan")
    n8 = quan.F8Rows(q.view(torch.float8_e4m3fn), scale, C)
    each = scale.repeat_interleave(128, dim=1)[:, :Q, :rows].permute(2, 0, 1)
    want = (n8.q.float()[:, :, :Q] * each).to(torch.bfloat16).reshape(rows, C)
    assert int(want.isnan().sum()) == Q - 128 * (blocks - 1)
    for shift in (0, 1):
        buf = torch.full((rows * C + 16,), 7.0, device="cuda", dtype=torch.bfloat16)
        out = buf[shift:shift + rows * C].view(rows, C)
        quan.dequantize_f8_rows(n8, out=out)
        assert torch.equal(out.nan_to_num(12345.0), want.nan_to_num(12345.0))
        assert (buf[:shift] == 7).all() and (buf[shift + rows * C:] == 7).all()
