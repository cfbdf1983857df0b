"""The distillation loss and its gradient on the GPU against the fp64 oracle.

Tolerances, from the arithmetic (u = 2^-24).  With x = (z - max) / T, a power 2^(x log2 e) has the
relative error |x| 2u of its rounded argument and 2^-22 of the instruction; weighted with the powers
themselves, |x| is at most ln V < 12.  Their sum is a chain of at most V / 128 + 32 terms a thread
and a tree.  So S, and lse past its own rounding, is right to R = 5e-6 + (V / 128 + 32) u.  A single
q_v has its own |x|, and where it is taken from lse the roundings of lse and z / T: 4u (|z| / T +
|lse| + |x|).  ln p and p likewise with the teacher's logits.  A gradient in bf16 is rounded once
more: 2^-8 of itself."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.distill import distill
from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield


def f64(t):
    return t.detach().double().cpu().numpy()


def dev(a, dtype, shift=0):
    """A tensor of `dtype` whose first element lies `shift` elements into its storage."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(dtype)
    buf = torch.empty(t.numel() + shift, dtype=dtype, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def make(rows, V, top, dtype="bf16", pad=0, tdtype=None, bits=64, shift=0, seed=0, ignored=0.2,
         spread=3.0):
    rng = np.random.default_rng(seed)
    teacher = spread * rng.normal(size=(rows, V))
    z = np.full((rows, V + pad), 7.0)  # the padding's values are not read
    z[:, :V] = 0.7 * teacher + rng.normal(size=(rows, V))
    index = np.stack([rng.permutation(V)[:top] if V <= 4096 else
                      rng.choice(V, size=top, replace=False) for _ in range(rows)])
    t = np.take_along_axis(teacher, index, 1)
    drop = rng.uniform(size=index.shape) < 0.1  # empty slots of several kinds
    index = np.where(drop, rng.choice([-1, -100, V, V + 3, 2 ** 31 - 1], size=index.shape), index)
    t = np.where(rng.uniform(size=t.shape) < 0.05, -np.inf, t)
    index[rng.uniform(size=rows) < ignored] = -1
    it = torch.from_numpy(index).to(torch.int64 if bits == 64 else torch.int32).cuda()
    return dict(z=dev(z, DT[dtype], shift), index=it, teacher=dev(t, DT[tdtype or dtype]),
                g=dev(rng.uniform(0.5, 1.5, rows) * np.where(rng.uniform(size=rows) < 0.1, 0, 1),
                      torch.float32), V=V, dtype=dtype)


def want(d, T, scale=1.0):
    z = f64(d["z"])[:, :d["V"]]
    t, index = f64(d["teacher"]), d["index"].cpu().numpy()
    with np.errstate(invalid="ignore"):
        loss, lse, dz, q, share = distill(z, index, t, scale * f64(d["g"]), T)
    R = 5e-6 + (d["V"] / 128 + 32) * U
    x = np.abs(z - z.max(axis=1, keepdims=True)) / T
    # |ln p| of the slots, and |x| of their classes, weighted with p
    valid = (index >= 0) & (index < d["V"]) & (t > -np.inf)
    tm = np.where(valid, t, -np.inf).max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        tx = np.where(valid, np.abs(t - tm) / T, 0.0)
    rel_p = R + 4 * U * (tx.max(axis=1) + 6.0)
    lnp = tx.max(axis=1) + np.log(256.0)
    some = valid.any(axis=1)
    x_slots = np.where(share > 0, share * x, 0.0).sum(axis=1)
    tol_loss = T * T * (R + 8 * U * (x_slots + np.abs(lse) + lnp) + rel_p * (
        x_slots + lnp + np.abs(lse))) * some + 2 * U * np.abs(loss)
    tol_lse = R + 2 * U * (np.abs(lse) + np.abs(z).max(axis=1) / T)
    rel_q = R + 4 * U * (np.abs(z) / T + np.abs(lse)[:, None] + x)
    g = np.abs(scale * f64(d["g"]))[:, None] * T * some[:, None]
    # (a power below the smallest normal number, 2^-126, becomes 0: 2^-126 of q, times g)
    tol_dz = g * (q * rel_q + share * rel_p[:, None] + 2.0 ** -126) + \
        (2 * U + HALF[d["dtype"]]) * np.abs(dz)
    return loss, lse, dz, tol_loss, tol_lse, tol_dz


def within(got, ref, tol, what):
    got = f64(got)
    assert np.isfinite(got).all(), what
    worst = np.max(np.abs(got - ref) - tol)
    assert worst <= 0.0, "%s: past the tolerance by %.3e" % (what, worst)


def check(d, T=1.0, scale=1.0):
    V, pad = d["V"], d["z"].shape[1] - d["V"]
    loss, lse, dz, tol_loss, tol_lse, tol_dz = want(d, T, scale)
    args = dict(classes=V, temperature=T)
    got, got_lse = quan.distill_loss(d["z"], d["index"], d["teacher"], **args)
    within(got, loss, tol_loss, "loss")
    within(got_lse, lse, tol_lse, "lse")
    grad = quan.distill_loss_backward(d["g"], d["z"], got_lse, d["index"], d["teacher"],
                                      scale=scale, **args)
    both = quan.distill_loss_and_gradient(d["z"], d["index"], d["teacher"], d["g"], scale=scale,
                                          **args)
    within(both[0], loss, tol_loss, "loss with gradient")
    for what, x in (("gradient", grad), ("gradient with loss", both[1])):
        assert not f64(x)[:, V:].any(), what + " of padding"
        within(x[:, :V], dz, tol_dz, what)
    assert pad == 0 or both[1].shape == d["z"].shape
    return got, got_lse, grad, both


SIZES = [(1, 1, 1), (3, 2, 2), (5, 3, 1), (7, 7, 7), (300, 8, 3), (129, 31, 20), (64, 32, 32),
         (1000, 100, 10), (33, 127, 64), (50, 256, 256), (20, 257, 100), (40, 1000, 50),
         (17, 1024, 1), (9, 2051, 13), (6, 4099, 256), (5, 8192, 64), (4, 10007, 50),
         (3, 32768, 64), (2, 65536, 32), (1, 65536, 32), (1, 100003, 200), (2, 131072, 8),
         (1, 300001, 17)]


@pytest.mark.parametrize("rows, V, top", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values(rows, V, top, dtype):
    check(make(rows, V, top, dtype, seed=V))


@pytest.mark.parametrize("rows, V, top", [(40, 5, 3), (60, 100, 10), (9, 1000, 20), (3, 9999, 40),
                                          (2, 70001, 30)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad, shift", [(1, 0), (2, 1), (3, 5), (0, 3), (8, 8)])
def test_padded_and_misaligned_rows(rows, V, top, dtype, pad, shift):
    check(make(rows, V, top, dtype, pad, shift=shift, seed=pad), T=2.0)


@pytest.mark.parametrize("T", [0.125, 0.5, 4.0, 100.0])
@pytest.mark.parametrize("rows, V", [(30, 50), (4, 5000)])
def test_temperatures_and_scale(rows, V, T):
    check(make(rows, V, 12, "f32", seed=1), T, scale=0.25)


@pytest.mark.parametrize("dtype, tdtype", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("V", [60, 3000])
def test_types_of_the_slots(dtype, tdtype, bits, V):
    check(make(21, V, 9, dtype, tdtype=tdtype, bits=bits, seed=2))


@pytest.mark.parametrize("V", [6, 90, 2000, 40000])
def test_a_class_in_several_slots(V):
    d = make(24, V, 5, "f32", seed=3, ignored=0.0)
    d["index"][:, 1:4] = d["index"][:, :1]
    d["index"][3] = V - 1
    d["index"][4] = 0
    check(d)


@pytest.mark.parametrize("V", [4, 90, 2000, 40000])
def test_classes_that_cannot_be(V):
    # logits of -infinity (a masked class) and of the type's lowest value: q = 0 there, no NaN
    for low in (-np.inf, float(torch.finfo(torch.bfloat16).min)):
        d = make(12, V, 2, "bf16", seed=4, ignored=0.0)
        slots = d["index"].clamp(0, V - 1).long()
        keep = torch.gather(d["z"], 1, slots)
        d["z"][:, ::2] = low
        d["z"].scatter_(1, slots, keep)  # (no slot's class is masked)
        if (torch.isinf(d["z"]).all(dim=1)).any():
            d["z"][:, 0] = 0.0
        got = quan.distill_loss_and_gradient(d["z"], d["index"], d["teacher"], d["g"])
        z = f64(d["z"])
        with np.errstate(invalid="ignore"):
            ref = distill(z, d["index"].cpu().numpy(), f64(d["teacher"]), f64(d["g"]))
        assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all()
        assert np.abs(f64(got[0]) - ref[0]).max() <= 1e-4 * max(1.0, np.abs(ref[0]).max())
        # (a bf16 rounding, and 1e-4 of q and of the shares, each at most 1)
        assert (np.abs(f64(got[1]) - ref[2]) <= 2.0 ** -8 * np.abs(ref[2]) + 1.5e-4).all()
        masked = (d["z"] == low) & (torch.from_numpy(ref[4]).cuda() == 0)
        assert not got[1][masked].any()


@pytest.mark.parametrize("V", [4, 90, 2000, 40000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), "none"])
def test_bad_logits_stay_in_their_row(V, bad):
    d = make(9, V, 3, "f32", seed=5, ignored=0.0)
    d["g"].fill_(0.5)
    d["index"][:, 0] = 0
    d["teacher"][:, 0] = 1.0
    args = (d["index"], d["teacher"])
    good = quan.distill_loss_and_gradient(d["z"], *args, d["g"])
    z = d["z"].clone()
    if bad == "none":
        z[4] = -float("inf")
    else:
        z[4, V // 2] = bad
    got = quan.distill_loss_and_gradient(z, *args, d["g"])
    loss, lse = quan.distill_loss(z, *args)
    keep = [r for r in range(9) if r != 4]
    assert torch.isnan(got[0][4]) and torch.isnan(got[1][4]).all() and torch.isnan(loss[4])
    assert torch.equal(got[0][keep], good[0][keep]) and torch.equal(got[1][keep], good[1][keep])
    grad = quan.distill_loss_backward(d["g"], z, lse, *args)
    assert torch.isnan(grad[4]).all() and torch.isfinite(grad[keep]).all()
    # no slots, or no weight: such a row has no part
    index, g = d["index"].clone(), d["g"].clone()
    index[4] = -1
    got = quan.distill_loss_and_gradient(z, index, d["teacher"], g)
    assert got[0][4] == 0 and not got[1][4].any()
    g[4] = 0
    grad = quan.distill_loss_backward(g, z, lse, *args)
    assert not grad[4].any() and not quan.distill_loss_and_gradient(z, *args, g)[1][4].any()


def test_an_impossible_class_that_is_wanted():
    d = make(2, 50, 3, "f32", seed=6, ignored=0.0)
    d["index"][:] = torch.tensor([1, 2, 3])
    d["teacher"].zero_()
    d["z"][0, 2] = -float("inf")
    loss, lse = quan.distill_loss(d["z"], d["index"], d["teacher"])
    assert loss[0] == float("inf") and torch.isfinite(loss[1]) and torch.isfinite(lse).all()
    grad = quan.distill_loss_backward(None, d["z"], lse, d["index"], d["teacher"])
    assert torch.isfinite(grad).all() and abs(float(grad[0, 2]) + 1 / 3) < 1e-6


@pytest.mark.parametrize("V", [10, 100, 3000, 70001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_repeats(V, dtype):
    d = make(37, V, 7, dtype, 3, seed=7)
    args = (d["index"], d["teacher"])
    loss, grad = quan.distill_loss_and_gradient(d["z"], *args, d["g"], classes=V)
    for _ in range(3):
        a, b = quan.distill_loss_and_gradient(d["z"], *args, d["g"], classes=V)
        assert torch.equal(a, loss) and torch.equal(b, grad)
    l2, lse = quan.distill_loss(d["z"], *args, classes=V)
    g2 = quan.distill_loss_backward(d["g"], d["z"], lse, *args, classes=V)
    z = d["z"].clone()
    assert quan.distill_loss_backward(d["g"], z, lse, *args, classes=V, out=z) is z
    assert torch.equal(z, g2)
    z = d["z"].clone()
    out = torch.empty_like(loss)
    a, b = quan.distill_loss_and_gradient(z, *args, d["g"], classes=V, out=z, loss=out)
    assert a is out and b is z and torch.equal(a, loss) and torch.equal(b, grad)


def test_weights_default_to_one():
    d = make(20, 64, 6, "f32", seed=8)
    _, lse = quan.distill_loss(d["z"], d["index"], d["teacher"])
    one = torch.ones(20, device="cuda")
    a = quan.distill_loss_backward(None, d["z"], lse, d["index"], d["teacher"])
    assert torch.equal(a, quan.distill_loss_backward(one, d["z"], lse, d["index"], d["teacher"]))
    a = quan.distill_loss_and_gradient(d["z"], d["index"], d["teacher"])[1]
    assert torch.equal(a, quan.distill_loss_and_gradient(d["z"], d["index"], d["teacher"], one)[1])


def test_leading_shape_streams_and_no_rows():
    d = make(60, 100, 5, seed=9)
    a = quan.distill_loss_and_gradient(d["z"], d["index"], d["teacher"], d["g"])
    args = (d["z"].view(3, 4, 5, 100), d["index"].view(3, 4, 5, 5), d["teacher"].view(3, 4, 5, 5),
            d["g"].view(3, 4, 5))
    b = quan.distill_loss_and_gradient(*args)
    assert b[0].shape == (3, 4, 5) and torch.equal(b[0].view(-1), a[0])
    assert torch.equal(b[1].view(60, 100), a[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        c = quan.distill_loss_and_gradient(*args, stream=stream)
        s.synchronize()
        assert torch.equal(c[0], b[0]) and torch.equal(c[1], b[1])
    e = [x[:0] for x in args]
    loss, dz = quan.distill_loss_and_gradient(*e)
    assert loss.shape == (0, 4, 5) and dz.shape == (0, 4, 5, 100)


@pytest.mark.parametrize("rows, V", [(50, 100), (3, 20000), (1, 65536)])
def test_captured(rows, V):
    d = make(rows, V, 5, "f32", seed=10, ignored=0.0)
    args = (d["z"], d["index"], d["teacher"], d["g"])
    quan.distill_loss_and_gradient(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        loss, lse = quan.distill_loss(*args[:3])
        grad = quan.distill_loss_backward(d["g"], d["z"], lse, d["index"], d["teacher"])
        both = quan.distill_loss_and_gradient(*args)
    for seed in (11, 12):
        new = make(rows, V, 5, "f32", seed=seed, ignored=0.0)
        for k in ("z", "index", "teacher", "g"):
            d[k].copy_(new[k])
        g.replay()
        torch.cuda.synchronize()
        want = quan.distill_loss_and_gradient(*args)
        l2, lse2 = quan.distill_loss(*args[:3])
        assert torch.equal(both[0], want[0]) and torch.equal(both[1], want[1])
        assert torch.equal(loss, l2) and torch.equal(lse, lse2)
        assert torch.equal(grad, quan.distill_loss_backward(d["g"], d["z"], lse2, d["index"],
                                                            d["teacher"]))


def test_past_two_to_the_31_logits():
    rows, V = 70000, 32768  # 2.3e9 logits, 4.6 GB
    z = torch.randn(rows, 64, device="cuda").to(torch.bfloat16).repeat(1, V // 64)
    index = torch.randint(0, V, (rows, 4), device="cuda")
    t = torch.randn(rows, 4, device="cuda")
    at = torch.tensor([0, 1, 32767, 65535, 65536, rows - 2, rows - 1], device="cuda")
    d = dict(z=z[at].clone(), index=index[at], teacher=t[at], V=V, dtype="bf16",
             g=torch.ones(7, device="cuda"))
    loss, lse, dz, tol_loss, tol_lse, tol_dz = want(d, 1.0)
    got, grad = quan.distill_loss_and_gradient(z, index, t, out=z)
    within(got[at], loss, tol_loss, "loss")
    within(grad[at], dz, tol_dz, "gradient")


def test_refuses_on_the_device():
    d = make(4, 20, 3, "f32")
    z, i, t = d["z"], d["index"], d["teacher"]
    with pytest.raises(ValueError, match="index must"):
        quan.distill_loss(z, i.float(), t)
    with pytest.raises(ValueError, match="index must"):
        quan.distill_loss(z, i[:2], t)
    with pytest.raises(ValueError, match="teacher must"):
        quan.distill_loss(z, i, t[:, :2])
    with pytest.raises(ValueError, match="logits must"):
        quan.distill_loss(z[:, ::2], i, t)
    with pytest.raises(ValueError, match="dloss must"):
        quan.distill_loss_and_gradient(z, i, t, torch.ones(3, device="cuda"))
    with pytest.raises(ValueError, match="out must"):
        quan.distill_loss_and_gradient(z, i, t, out=z.to(torch.bfloat16))
    with pytest.raises(quan.QuanError):
        quan.distill_loss(z, i, t, classes=21)
    with pytest.raises(quan.QuanError):
        quan.distill_loss(z, i, t, temperature=0.0)
    with pytest.raises(quan.QuanError):
        quan.distill_loss_and_gradient(z, i, t, out=z, loss=z.view(-1)[:4])


def reference(d, T):
    """The oracle's arithmetic for many rows at once, in fp64 on the device."""
    V, index = d["V"], d["index"].long()
    z, t = d["z"][:, :V].double() / T, d["teacher"].double() / T
    valid = (index >= 0) & (index < V) & (t > -float("inf"))
    some = valid.any(dim=1, keepdim=True)
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    logp = torch.log_softmax(torch.where(valid | ~some, t.clamp(min=-1e300), -1e300), dim=1)
    p = torch.where(valid, logp.exp(), 0.0)
    at = torch.where(valid, index, 0)
    loss = T * T * torch.where(p > 0, p * (logp - (z.gather(1, at) - lse)), 0.0).sum(dim=1)
    share = torch.zeros_like(z).scatter_add_(1, at, p)
    q = (z - lse).exp()
    return loss, lse[:, 0], torch.where(some, T * d["g"].double()[:, None] * (q - share), 0.0), q, share


MANY = [(3000, 5, 0, 2), (3000, 100, 1, 10), (2500, 513, 0, 40), (2500, 1023, 3, 100),
        (2000, 2046, 2, 64), (2000, 2048, 0, 256), (2000, 2049, 0, 5), (3000, 2549, 2, 123),
        (3000, 4246, 3, 20), (2600, 6633, 0, 11), (1300, 8192, 0, 30), (1300, 11321, 0, 4),
        (700, 16384, 1, 8), (700, 20000, 0, 33), (500, 27855, 2, 27), (500, 32768, 0, 64),
        (400, 32767, 1, 64), (200, 70003, 0, 9)]


@pytest.mark.parametrize("rows, V, pad, top", MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(rows, V, pad, top, dtype):
    # more rows than a block of any kind takes at once, of every length that picks another kernel
    T = 2.0
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.full((rows, V + pad), 9.0, device="cuda", dtype=DT[dtype])
    z[:, :V] = 3.0 * torch.randn(rows, V, generator=g, device="cuda")
    # rows of different magnitudes and offsets: what one leaves behind would show in another
    z[:, :V] *= torch.rand(rows, 1, generator=g, device="cuda") * 2
    z[:, :V] += 40.0 * torch.randn(rows, 1, generator=g, device="cuda")
    index = torch.randint(0, V, (rows, top), generator=g, device="cuda")
    index[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    t = torch.randn(rows, top, generator=g, device="cuda").to(DT[dtype])
    d = dict(z=z, index=index, teacher=t, V=V, dtype=dtype,
             g=torch.rand(rows, generator=g, device="cuda") + 0.5)
    loss, lse, dz, q, share = reference(d, T)
    args = dict(classes=V, temperature=T)
    l1, e1 = quan.distill_loss(z, index, t, **args)
    g1 = quan.distill_loss_backward(d["g"], z, e1, index, t, **args)
    l2, g2 = quan.distill_loss_and_gradient(z, index, t, d["g"], **args)
    R = 5e-6 + (V / 128 + 32) * U
    x = (z[:, :V].double().amax(dim=1) / T).abs() + lse.abs() + 30.0  # |x| of what counts
    for got in (l1, l2):
        assert ((got.double() - loss).abs() <= T * T * 2 * (R + 16 * U * x) * (1 + loss / T / T)).all()
    assert ((e1.double() - lse).abs() <= R + 4 * U * x).all()
    for got in (g1, g2):
        assert not got[:, V:].any()
        tol = T * d["g"].double()[:, None] * (q + share) * (R + 8 * U * (x + 60.0))[:, None]
        assert ((got[:, :V].double() - dz).abs() <= tol + HALF[dtype] * dz.abs() + 1e-30).all()


@pytest.mark.parametrize("rows, V", [(50, 8), (50, 64), (20, 256), (4000, 100)])
@pytest.mark.parametrize("T", [1.0, 4.0])
def test_a_student_like_its_teacher(rows, V, T):
    # every class a slot, with the student's own logit: the loss is 0 and the gradient too.  Both sums
    # have the same terms, at most (V / 4 + 8) roundings apart; ln p and ln q differ by four roundings
    # of at most |x| + ln V, |x| < 20
    z = torch.randn(rows, V, device="cuda") * 2
    index = torch.argsort(torch.rand(rows, V, device="cuda"), dim=1)
    t = z.gather(1, index)
    loss, dz = quan.distill_loss_and_gradient(z, index, t, temperature=T)
    tol = 2 * (V / 4 + 8) * U + 4 * U * (20 / T + np.log(V))
    assert loss.abs().max() <= T * T * tol and dz.abs().max() <= T * 2 * tol
    l2, lse = quan.distill_loss(z, index, t, temperature=T)
    assert l2.abs().max() <= T * T * tol


@pytest.mark.parametrize("V", [90, 2000, 5000, 12000, 32000, 70001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_classes_of_rows_far_below_zero(V, dtype):
    # all but 64 classes masked, so that most threads see no finite logit, and a largest logit whose
    # distance from 0 no fp32 power spans; with a row of one class, and one that has none
    rows, top, keep = 320, 6, 64
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.full((rows, V), -float("inf"), device="cuda")
    z[:, :keep] = 3.0 * torch.randn(rows, keep, generator=g, device="cuda") - 400.0
    z[5, 1:] = -float("inf")
    z[6] = -float("inf")
    z = z.to(DT[dtype])
    index = torch.randint(0, keep, (rows, top), generator=g, device="cuda")
    index[5], index[6] = 0, -1
    d = dict(z=z, index=index, teacher=torch.randn(rows, top, generator=g, device="cuda"), V=V,
             g=torch.rand(rows, generator=g, device="cuda") + 0.5)
    loss, lse, dz, q, share = reference(d, 1.0)
    loss[6], lse[6], dz[6], q[6] = 0.0, -float("inf"), 0.0, 0.0
    l1, e1 = quan.distill_loss(z, index, d["teacher"])
    g1 = quan.distill_loss_backward(d["g"], z, e1, index, d["teacher"])
    l2, g2 = quan.distill_loss_and_gradient(z, index, d["teacher"], d["g"])
    # (as above: roundings of logits and sums of up to 400 + 30)
    R = 5e-6 + (V / 128 + 32) * U + 16 * U * 860.0
    # (relative to its magnitude: a row whose slots all have its one possible class, as row 5, has
    # ln q = 0 and the loss sum p ln p, at least -ln 6)
    for got in (l1, l2):
        assert ((got.double() - loss).abs() <= 2 * R * (1 + loss.abs())).all()
    assert e1[6] == -float("inf")
    others = torch.arange(rows, device="cuda") != 6
    assert ((e1.double() - lse).abs()[others] <= R).all()
    for got in (g1, g2):
        tol = d["g"].double()[:, None] * (q + share) * R + HALF[dtype] * dz.abs() + 1e-30
        assert ((got.double() - dz).abs() <= tol).all()
        assert not got[:, keep:].any()


@pytest.mark.parametrize("rows, V, pad, top", [(320, 70001, 0, 5), (310, 33001, 3, 20),
                                               (160, 40000, 8, 64), (1500, 2500, 1, 256),
                                               (5000, 4100, 4, 3), (1300, 16390, 2, 40),
                                               (700, 14001, 1, 50), (640, 30001, 0, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_more_lengths(rows, V, pad, top, dtype):
    test_many_rows(rows, V, pad, top, dtype)
