"""The residual mixing stack on the GPU: every step of a training pass against the fp64 oracle,
from the tensors that the pass itself kept (so each is held to its own operator's rounding), a
captured step that draws new masks, and a short run that learns."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks
from paper_2509_05512_gb300 import build, quan
from paper_2509_05512_gb300.mixer import Mixer, train

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield
    assert quan.quan_device_status()[0] == quan.QUAN_OK


def rows(t):
    return t.double().cpu().numpy().reshape(-1, t.shape[-1])


def near(got, want, what):
    # one bf16 rounding of an fp32 result: 2^-8 of the element, and sums below 1e-5 of the
    # largest term, taken as the largest result of the row (no cancellation in these inputs)
    got = rows(got)
    tol = 2.0 ** -8 * np.abs(want) + 2e-4 * np.abs(want).max(axis=1, keepdims=True)
    assert (np.abs(got - want) <= tol).all(), what


def test_one_training_pass():
    N, H, C, depth, p = 3, 9, 96, 2, 0.25
    m = Mixer(C, depth, p=p, alpha=0.5, seed=7)
    m.counter.fill_(1000)
    x = torch.randn(N, H, H, C, device="cuda").to(torch.bfloat16)
    dn = torch.randn(N, H, H, C, device="cuda").to(torch.bfloat16)
    out = m.forward(x)
    assert out is m.n[-1]
    grads = m.backward(dn)
    per = -(-x.numel() // 8)
    ones = np.ones(C)
    near(m.n[0], blocks.join(rows(x), pre=ones, groups=4)[1], "n 0")
    kw = [dict(post=ones, gate=0.5 * ones, pre=ones, alpha=0.5, groups=4,
               factor=blocks.dropout_factor(x.numel(), p, 7, 1000 + l * per).reshape(-1, C))
          for l in range(depth)]
    for l in range(depth):
        letters = [blocks.f8_letter(w.double().cpu().numpy()[:, 0, 0])[0] for w in m.letters[l]]
        near(m.h[l], blocks.qpoint(blocks.f8_rows(rows(m.n[l])), letters)[0], "h %d" % l)
        y, n = blocks.join(rows(m.y[l]), rows(m.h[l]), **kw[l])
        near(m.y[l + 1], y, "y %d" % l)
        near(m.n[l + 1], n, "n %d" % (l + 1))
    # the gradients of the last block, from what it was given
    want = blocks.join_backward(None, rows(dn), rows(m.y[depth]), rows(m.h[depth - 1]),
                                **kw[depth - 1])
    for name, w in (("post", want[2]), ("gate", want[3])):
        g = grads[name][depth - 1].double().cpu().numpy()
        assert np.linalg.norm(g - w) <= 1e-4 * np.linalg.norm(w), name
    g = grads["pre"][depth].double().cpu().numpy()
    assert np.linalg.norm(g - want[4]) <= 1e-4 * np.linalg.norm(want[4])
    assert grads["dx"].shape == x.shape and len(grads["letters"]) == depth
    assert all(d.shape == (C // 4, 1, 1, C // 4) and d.dtype == torch.float32
               for block in grads["letters"] for d in block)


def test_captured_step_draws_new_masks():
    m = Mixer(64, 2, p=0.5, seed=3)
    x = torch.randn(2, 8, 8, 64, device="cuda").to(torch.bfloat16)
    dn = torch.randn_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.forward(x)
        m.backward(dn)
    torch.cuda.synchronize()
    m.counter.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = m.forward(x)
        m.backward(dn)
        m.advance()
    seen = []
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        seen.append(out.clone())
    assert int(m.counter) == 3 * 2 * (x.numel() // 8)
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])
    m.counter.zero_()
    assert torch.equal(m.forward(x), seen[0])


def test_training_learns():
    losses = train(steps=25, N=2, H=8, channels=64, depth=2, report=None)
    assert np.isfinite(losses).all() and losses[-1] < 0.8 * losses[0]
