"""The mixing stack trained by distillation and served with 4-bit letters: the new operators as they
are used together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.distill import distill
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer, distillation, train

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
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("groups", [1, 4])
def test_a_step_and_serving(groups):
    N, H, C, top, T = 2, 5, 128, 7, 2.0
    m = Mixer(C, 2, groups=groups, p=0.25, seed=4)
    x = torch.randn(N, H, H, C, device="cuda").to(torch.bfloat16)
    index = torch.stack([torch.randperm(C, device="cuda")[:top] for _ in range(N * H * H)])
    index = index.view(N, H, H, top)
    index[0, 0] = -1  # pixels without a label
    teacher = torch.randn(N, H, H, top, device="cuda")
    loss, dn = distillation(m, x, index, teacher, temperature=T)
    weight = np.full(N * H * H, 1.0 / (N * H * H - H))
    weight[:H] = 0.0
    rows = lambda t: f64(t).reshape(N * H * H, -1)
    want, _, dz, _, _ = distill(rows(m.n[-1]), index.cpu().numpy().reshape(-1, top), rows(teacher),
                                weight, T)
    assert abs(float(loss) - (want * weight).sum()) <= 1e-4 * float(loss)
    # one bf16 rounding, and 1e-4 of a share of one pixel
    assert (np.abs(rows(dn) - dz) <= 2.0 ** -8 * np.abs(dz) + 1e-4 * T * weight.max()).all()
    grads = m.backward(dn)
    assert grads["dx"].shape == x.shape and torch.isfinite(grads["dx"]).all()
    m.update(grads, 0.1)
    m.quantize_4bit(group=32)
    one = x[:1, :1, :1].contiguous()
    out = m.serve(one)
    assert out.shape == one.shape and torch.isfinite(out).all()


def test_the_gradient_through_the_stack_is_the_loss_difference():
    # in the last norm's gain, which acts behind all quantisation: the loss's difference along it
    m = Mixer(64, 1, seed=5)
    x = torch.randn(1, 6, 6, 64, device="cuda").to(torch.bfloat16)
    index = torch.randint(0, 64, (1, 6, 6, 4), device="cuda")
    teacher = torch.randn(1, 6, 6, 4, device="cuda")
    d = torch.randn(64, device="cuda")
    _, dn = distillation(m, x, index, teacher, training=False)
    slope = float((m.backward(dn)["pre"][1] * d).sum())

    def loss(step):
        keep = m.pre[1].clone()
        m.pre[1] += step * d
        out = m.forward(x, training=False)
        z = f64(quan.residual_join(m.y[1], pre=m.pre[1], groups=4, eps=m.eps)[1]).reshape(36, 64)
        m.pre[1].copy_(keep)
        del out
        w = np.full(36, 1.0 / 36)
        return w @ distill(z, index.cpu().numpy().reshape(36, 4), f64(teacher).reshape(36, 4), w)[0]

    # logits are rounded to bf16 (2^-8 of values up to 4): 36 x 64 such errors of 0.01 at random move
    # the mean loss by less than 3e-4, which the step of 0.2 divides; a curvature below 1 adds
    # 0.2^2 / 6 of the third derivative
    got = (loss(0.1) - loss(-0.1)) / 0.2
    assert abs(got - slope) <= 3e-3 + 0.02 * abs(slope)


def test_training_by_distillation_runs():
    losses = train(steps=3, N=2, H=8, channels=64, depth=2, top=5, temperature=2.0, report=None)
    assert len(losses) == 3 and np.isfinite(losses).all()


def test_captured_step():
    m = Mixer(64, 2, p=0.5, seed=3)
    x = torch.randn(2, 8, 8, 64, device="cuda").to(torch.bfloat16)
    index = torch.randint(0, 64, (2, 8, 8, 4), device="cuda")
    teacher = torch.randn(2, 8, 8, 4, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        distillation(m, x, index, teacher)
    torch.cuda.synchronize()
    m.counter.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        loss, dn = distillation(m, x, index, teacher)
        m.advance()
    seen = []
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        seen.append((float(loss), dn.clone()))
    assert seen[0][0] != seen[1][0]
    m.counter.zero_()
    loss, dn = distillation(m, x, index, teacher)
    assert float(loss) == seen[0][0] and torch.equal(dn, seen[0][1])


def test_pixels_without_a_slot_in_use_have_no_part_in_the_mean():
    # however a slot is left empty: no class, a class past the channels, a teacher that gives it nothing
    m = Mixer(64, 1, seed=6)
    x = torch.randn(1, 4, 4, 64, device="cuda").to(torch.bfloat16)
    index = torch.randint(0, 64, (1, 4, 4, 3), device="cuda")
    teacher = torch.randn(1, 4, 4, 3, device="cuda")
    seen = []
    for empty in range(3):
        i, t = index.clone(), teacher.clone()
        if empty == 0:
            i[0, 1] = -1
        elif empty == 1:
            i[0, 1] = 64
        else:
            t[0, 1] = -float("inf")
        loss, dn = distillation(m, x, i, t, training=False)
        seen.append((float(loss), dn.clone()))
    assert not seen[0][1][0, 1].any()
    for loss, dn in seen[1:]:
        assert loss == seen[0][0] and torch.equal(dn, seen[0][1])
