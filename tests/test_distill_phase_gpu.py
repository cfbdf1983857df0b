"""The distillation loss where logits and gradient do not begin on the same 16-byte phase, in every
kernel; and the two ways to a gradient for logits far from 0.  Tolerances as in test_distill_gpu.py."""
import pytest

torch = pytest.importorskip("torch")

from paper_2509_05512_gb300 import build, quan
from test_distill_gpu import DT, HALF, U, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield


def shifted(shape, dtype, shift, fill=float("nan")):
    """(a tensor whose first element lies `shift` elements into its storage, that storage, its end)."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((shift + n + 8,), fill, dtype=dtype, device="cuda")
    return buf[shift:shift + n].view(shape), buf, shift + n


def make(rows, V, pad, top, dtype, shift, offset=0.0):
    g = torch.Generator(device="cuda").manual_seed(V + shift)
    z, _, _ = shifted((rows, V + pad), DT[dtype], shift)
    z.fill_(9.0)  # the padding's values are not read
    z[:, :V] = 3.0 * torch.randn(rows, V, generator=g, device="cuda") + offset
    index = torch.randint(0, V, (rows, top), generator=g, device="cuda")
    index[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    return dict(z=z, index=index, V=V, dtype=dtype,
                teacher=torch.randn(rows, top, generator=g, device="cuda").to(DT[dtype]),
                g=torch.rand(rows, generator=g, device="cuda") + 0.5)


def bound(d, T, q, share, dz, lse, from_lse):
    """How far a gradient may be off: sums and powers, and where q is taken from lse the roundings of
    z / T and lse."""
    z = d["z"][:, :d["V"]].double()
    x = (z - z.amax(dim=1, keepdim=True)).abs() / T
    rel_q = 5e-6 + (d["V"] / 128 + 32) * U + 4 * U * x
    if from_lse:
        rel_q = rel_q + 4 * U * (z.abs() / T + lse[:, None].abs())
    t = d["teacher"].double()
    rel_p = 5e-6 + 32 * U + 4 * U * ((t.amax(dim=1) - t.amin(dim=1)) / T + 6.0)
    g = T * d["g"].double()[:, None]
    return g * (q * rel_q + share * rel_p[:, None] + 2.0 ** -126) + (2 * U + HALF[d["dtype"]]) * dz.abs()


# rows of a tile, of the ring with 128, 256 and 512 threads, of the ring for the gradient alone (48 to
# 64 KB, 608 rows or more), and of blocks that share a row
SIZES = [(300, 60, 1, 7, "bf16"), (300, 60, 0, 7, "f32"), (700, 3000, 0, 20, "bf16"),
         (700, 3001, 1, 256, "f32"), (700, 9000, 1, 20, "bf16"), (700, 9001, 0, 20, "f32"),
         (700, 30000, 1, 20, "bf16"), (700, 15000, 3, 20, "f32"), (20, 70001, 1, 9, "bf16"),
         (40, 9000, 1, 9, "f32")]


@pytest.mark.parametrize("rows, V, pad, top, dtype", SIZES)
@pytest.mark.parametrize("shift, out_shift", [(1, 0), (3, 0), (0, 1), (3, 6), (2, 3)])
def test_gradient_on_another_phase(rows, V, pad, top, dtype, shift, out_shift):
    T, d = 2.0, make(rows, V, pad, top, dtype, shift)
    args, kw = (d["index"], d["teacher"]), dict(classes=V, temperature=T)
    loss, lse, dz, q, share = reference(d, T)
    l1, e1 = quan.distill_loss(d["z"], *args, **kw)
    x = (d["z"][:, :V].double().amax(dim=1) / T).abs() + lse.abs() + 30.0  # |x| of what counts
    R = 5e-6 + (V / 128 + 32) * U
    tol_loss = T * T * 2 * (R + 16 * U * x) * (1 + loss / T / T)
    assert ((l1.double() - loss).abs() <= tol_loss).all()
    found = []
    for at in (out_shift, None):  # None: left to the call, on 16 bytes
        for both in (False, True):
            out, buf, end = shifted(d["z"].shape, DT[dtype], at or 0, fill=123.0)
            given = None if at is None else out
            if both:
                l2, got = quan.distill_loss_and_gradient(d["z"], *args, d["g"], out=given, **kw)
                assert ((l2.double() - loss).abs() <= tol_loss).all()
            else:
                got = quan.distill_loss_backward(d["g"], d["z"], e1, *args, out=given, **kw)
            if given is not None:
                assert got is out
                # nothing beside it is written
                assert (buf[:at] == 123.0).all() and (buf[end:] == 123.0).all()
            assert not got[:, V:].any()
            tol = bound(d, T, q, share, dz, lse, not both)
            assert ((got[:, :V].double() - dz).abs() <= tol).all()
            found.append(got)
    # the same values wherever they are written
    assert torch.equal(found[0], found[2]) and torch.equal(found[1], found[3])


@pytest.mark.parametrize("rows, V", [(200, 60), (700, 3000), (700, 15000), (5, 40000)])
@pytest.mark.parametrize("offset, T", [(5000.0, 1.0), (-5000.0, 1.0), (20.0, 0.005)])
def test_logits_far_from_zero(rows, V, offset, T):
    # q from lse, one fp32 number, carries lse's rounding into the whole row: off by about
    # 2^-23 (|z| / T + |lse|) of itself.  The call that has the row's maximum has no such term.
    d = make(rows, V, 0, 9, "f32", 0, offset)
    args, kw = (d["index"], d["teacher"]), dict(temperature=T)
    loss, lse, dz, q, share = reference(d, T)
    _, e1 = quan.distill_loss(d["z"], *args, **kw)
    alone = quan.distill_loss_backward(d["g"], d["z"], e1, *args, **kw)
    _, both = quan.distill_loss_and_gradient(d["z"], *args, d["g"], **kw)
    for got, from_lse in ((alone, True), (both, False)):
        tol = bound(d, T, q, share, dz, lse, from_lse)
        assert ((got.double() - dz).abs() <= tol).all()
