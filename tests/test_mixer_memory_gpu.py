"""What one forward pass of the mixing stack allocates."""
import pytest

torch = pytest.importorskip("torch")

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


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("channels, depth", [(256, 1), (256, 4), (244, 3), (64, 3)])
def test_a_block_allocates_no_more_than_its_tensors_and_a_workspace(groups, channels, depth):
    # small passes are host time, and an allocation between launches is 2 to 5 us of it: the first norm,
    # then y, n, h and one workspace a block, be it the product's or rows in 8 bits
    m = Mixer(channels, depth, groups=groups, p=0.1)
    x = torch.randn(8, 16, 16, channels, device="cuda").to(torch.bfloat16)
    count = lambda: torch.cuda.memory_stats()["allocation.all.allocated"]
    m.forward(x)
    m.forward(x)
    before = count()
    m.forward(x)
    # (rows in 8 bits are two tensors, which the blocks share)
    assert count() - before <= 1 + 4 * depth + (groups == 4 and depth == 1)


def test_blocks_that_share_their_rows_give_what_rows_of_their_own_give():
    m = Mixer(244, 4, p=0.1, seed=2)
    x = torch.randn(4, 9, 9, 244, device="cuda").to(torch.bfloat16)
    out = m.forward(x)
    _, n, rows = quan.residual_join_f8(x, pre=m.pre[0], groups=4, eps=m.eps, keep=True)
    y = x
    for l in range(4):
        h = quan.qpointwise_f8(rows, m.w[l])
        y, n, rows = quan.residual_join_f8(y, h, keep=True, **m._join(l, x.numel(), True))
    assert torch.equal(out, n)
