"""The 8-bit pointwise product on the GPU against the fp64 oracle.

Quantisation has one right answer, so the 8-bit letters and their scales are compared bit for
bit.  An output is a sum of exact products taken in fp32 (at most 128 in the tensor cores'
accumulators, then chains of blocks, and the epilogue's few roundings) and rounded once to bf16:
within 2^-8 of itself and 2e-5 of the sum of its terms' magnitudes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu

ACT = {"none": quan.QUAN_ACT_NONE, "relu": quan.QUAN_ACT_RELU, "silu": quan.QUAN_ACT_SILU}


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


def bf16(a, shift=0):
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(torch.bfloat16)
    buf = torch.empty(t.numel() + shift, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def letters(Cin, Cout, seed):
    rng = np.random.default_rng(seed)
    # blocks of different magnitudes
    mag = np.exp2(rng.integers(-3, 4, size=(4, Cout // 4, 1)))
    return [bf16(rng.normal(size=(Cout // 4, 1, 1, Cin // 4)) * mag[k][:, :, None, None] /
                 np.sqrt(Cin)) for k in range(4)]


def activations(rows, C, seed, shift=0):
    rng = np.random.default_rng(seed)
    return bf16(rng.normal(size=(rows, C)) * np.exp(rng.normal(size=C)) *
                np.exp2(rng.integers(-4, 5, size=(rows, 1))), shift)


def quantised(w):
    return [blocks.f8_letter(f64(v)[:, 0, 0])[0] for v in w]


def close(got, want, mag, what=""):
    got = f64(got).reshape(want.shape)
    assert np.isfinite(got).all(), what
    worst = np.max(np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 2e-5 * mag))
    assert worst <= 0.0, "%s: past the tolerance by %.3e" % (what, worst)


def check(rows, Cin, Cout, backward=False, act="none", vectors=(), seed=0, shift=0):
    w = letters(Cin, Cout, seed)
    x = activations(rows, Cout if backward else Cin, seed + 1, shift)
    f = quan.quantize_f8_weights(*w, transpose=backward)
    want, mag = blocks.qpoint(blocks.f8_rows(f64(x)), quantised(w), transpose=backward)
    if backward:
        got = quan.qpointwise_f8_backward_data(x, f)
        close(got, want, mag, "dx")
        return x, f, got
    rng = np.random.default_rng(seed + 2)
    v = {k: torch.from_numpy(rng.uniform(0.5, 1.5, Cout).astype(np.float32)).cuda()
         for k in vectors}
    got = quan.qpointwise_f8(x, f, act=ACT[act], **v)
    z, m = want, mag
    if "bias" in v:
        z, m = z + f64(v["bias"]), m + f64(v["bias"])
    if "scale" in v:
        z, m = z * f64(v["scale"]) + f64(v["shift"]), m * f64(v["scale"]) + f64(v["shift"])
    if act == "relu":
        z = np.maximum(z, 0.0)
    elif act == "silu":
        z = z / (1.0 + np.exp(-z))
    close(got, z, m, "y")
    return x, f, got


@pytest.mark.parametrize("Cin, Cout", [(4, 4), (64, 64), (520, 328), (512, 1024), (36, 2052),
                                       (1100, 516)])
@pytest.mark.parametrize("transpose", [False, True])
def test_letters(Cin, Cout, transpose):
    w = letters(Cin, Cout, 3)
    f = quan.quantize_f8_weights(*w, transpose=transpose)
    assert (f.Cin, f.Cout, f.transposed) == (Cin, Cout, transpose)
    q, s = f64(f.q.float()), f64(f.scale)
    n, k = (Cin // 4, Cout // 4) if transpose else (Cout // 4, Cin // 4)
    assert q.shape == (4, n, (k + 15) // 16 * 16) and not q[:, :, k:].any()
    for L in range(4):
        want, ws = blocks.f8_letter(f64(w[L])[:, 0, 0])
        want, ws = (want.T, ws.T) if transpose else (want, ws)
        assert np.array_equal(s[L], ws)
        each = np.repeat(np.repeat(ws, 128, 0), 128, 1)[:n, :k]
        assert np.array_equal(q[L, :, :k] * each, want)


SHAPES = [(1, 4, 4), (1, 512, 1024), (2, 64, 512), (3, 520, 36), (5, 1024, 1024), (8, 2048, 128),
          (17, 100, 340), (49, 2048, 512), (127, 512, 256), (128, 512, 256), (129, 512, 260),
          (1000, 328, 520), (777, 1028, 516), (300, 4, 2048), (640, 64, 64), (2500, 128, 1280),
          (20001, 256, 64), (20003, 1100, 64), (25000, 300, 20), (21000, 1028, 128),
          (20100, 516, 1032), (6000, 12, 28), (3000, 140, 44), (9000, 520, 264),
          (1280, 2060, 1024), (40000, 1032, 128), (16, 512, 512), (24, 2048, 512)]


@pytest.mark.parametrize("rows, Cin, Cout", SHAPES)
def test_product(rows, Cin, Cout):
    check(rows, Cin, Cout)


@pytest.mark.parametrize("rows, Cin, Cout", SHAPES)
def test_input_gradient(rows, Cin, Cout):
    check(rows, Cin, Cout, backward=True, seed=7)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("vectors", [(), ("bias",), ("scale", "shift"),
                                     ("bias", "scale", "shift")])
@pytest.mark.parametrize("rows, Cin, Cout", [(3, 256, 132), (300, 520, 640)])
def test_epilogue(rows, Cin, Cout, vectors, act):
    check(rows, Cin, Cout, act=act, vectors=vectors, seed=11)


@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("rows", [2, 200])
def test_misaligned_input_and_output(rows, shift):
    x, f, got = check(rows, 256, 512, shift=shift, seed=5)
    buf = torch.empty(got.numel() + shift, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:].view(got.shape)
    assert quan.qpointwise_f8(x, f, out=out) is out and torch.equal(out, got)


def test_every_product_of_the_hamilton_table():
    # one input and one output quaternion channel: the sixteen signed letters, both directions
    w = [bf16(np.full((1, 1, 1, 1), v)) for v in (1.0, 2.0, 4.0, 8.0)]
    eye = bf16(np.eye(4))
    y = f64(quan.qpointwise_f8(eye, quan.quantize_f8_weights(*w)))
    r, i, j, k = 1.0, 2.0, 4.0, 8.0
    block = np.array([[r, -i, -j, -k], [i, r, -k, j], [j, k, r, -i], [k, -j, i, r]])
    assert np.array_equal(y, block.T)
    dx = f64(quan.qpointwise_f8_backward_data(
        eye, quan.quantize_f8_weights(*w, transpose=True)))
    assert np.array_equal(dx, block)


@pytest.mark.parametrize("rows", [3, 300])
def test_zero_tiny_and_huge_blocks(rows):
    w = letters(1024, 256, 1)
    a = f64(activations(rows, 1024, 2))
    a[:, 128:256] = 0.0             # a block of zeros
    a[0] = 0.0                      # a row of zeros
    a[1, :128] *= 2.0 ** -130       # below the smallest scale: rounds to nothing
    a[2, 256:384] *= 2.0 ** 90
    x = bf16(a)
    got = quan.qpointwise_f8(x, quan.quantize_f8_weights(*w))
    want, mag = blocks.qpoint(blocks.f8_rows(f64(x)), quantised(w))
    close(got, want, mag)
    assert not got[0].any()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("rows", [4, 300])
def test_infinity_or_nan_makes_its_outputs_nan(rows, bad):
    w = letters(1024, 1024, 1)
    a = f64(activations(rows, 1024, 2))
    good = quan.qpointwise_f8(bf16(a), quan.quantize_f8_weights(*w), act=ACT["relu"])
    a[2, 700] = bad
    got = quan.qpointwise_f8(bf16(a), quan.quantize_f8_weights(*w), act=ACT["relu"])
    assert bool(torch.isnan(got[2]).all())
    keep = [r for r in range(rows) if r != 2]
    assert torch.equal(got[keep], good[keep])
    # a letter's block: the outputs of its 128 channels in the four components, no others
    w[1][130, 0, 0, 5] = bad
    a[2, 700] = 1.0
    got = f64(quan.qpointwise_f8(bf16(a), quan.quantize_f8_weights(*w)))
    hit = np.zeros((4, 256), dtype=bool)
    hit[:, 128:256] = True
    assert np.array_equal(np.isnan(got), np.broadcast_to(hit.reshape(-1), got.shape))


def test_workspace_streams_and_repeats():
    for rows in (2, 30, 1500):
        x, f, got = check(rows, 1024, 512, seed=9)
        need = quan.quan_qpoint_f8_workspace_size(rows, 1024, 512)
        ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for stream in (None, s, s.cuda_stream):
            again = quan.qpointwise_f8(x, f, stream=stream)
            s.synchronize()
            torch.cuda.synchronize()
            assert torch.equal(again, got)
        assert torch.equal(quan.qpointwise_f8(x, f, workspace=ws), got)  # whatever it held


def test_leading_shape_and_no_rows():
    x, f, got = check(60, 64, 128, seed=4)
    y = quan.qpointwise_f8(x.view(3, 4, 5, 64), f)
    assert y.shape == (3, 4, 5, 128) and torch.equal(y.view(60, 128), got)
    e = torch.empty((0, 4, 5, 64), dtype=torch.bfloat16, device="cuda")
    assert quan.qpointwise_f8(e, f).shape == (0, 4, 5, 128)


def test_output_past_two_to_the_31_elements():
    rows, Cin, Cout = 524300, 64, 4096  # 2.1e9 outputs, 4.3 GB
    w = letters(Cin, Cout, 2)
    f = quan.quantize_f8_weights(*w)
    x = torch.randn(rows, Cin, device="cuda").to(torch.bfloat16)
    got = quan.qpointwise_f8(x, f)
    at = torch.tensor([0, 1, 131071, 262143, 524287, 524288, rows - 2, rows - 1], device="cuda")
    want, mag = blocks.qpoint(blocks.f8_rows(f64(x[at])), quantised(w))
    close(got[at], want, mag)


def test_refuses_on_the_device():
    _, f, _ = check(2, 64, 64)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="x must"):
        quan.qpointwise_f8(x.float(), f)
    with pytest.raises(ValueError, match="x must"):
        quan.qpointwise_f8(x[:, :32], f)
    with pytest.raises(ValueError, match="bias"):
        quan.qpointwise_f8(x, f, bias=torch.zeros(32, device="cuda"))
    with pytest.raises(quan.QuanError):
        quan.qpointwise_f8(x, f, scale=torch.ones(64, device="cuda"))  # no shift
    with pytest.raises(quan.QuanError):
        quan.qpointwise_f8(x, f, out=x)


def test_bounded_waits_report_a_timeout():
    # the issuer waits on a barrier that nothing arrives on: every role gives up after the limit,
    # the status says so, and the next call is right again
    x, f, got = check(300, 512, 512, seed=8)
    quan.quan_set_wait_limit_ns(20_000_000)
    quan.quan_set_fault_injection(True)
    try:
        quan.qpointwise_f8(x, f)
        st, bits = quan.quan_device_status()
    finally:
        quan.quan_set_fault_injection(False)
        quan.quan_set_wait_limit_ns(0)
    assert st == quan.QUAN_ERR_DEVICE_TIMEOUT and bits != 0
    assert torch.equal(quan.qpointwise_f8(x, f), got)
    assert quan.quan_device_status()[0] == quan.QUAN_OK
