"""The residual block's Python helpers on the GPU: buffers that a caller gives, streams."""
import pytest

torch = pytest.importorskip("torch")

from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield
    assert quan.quan_device_status()[0] == quan.QUAN_OK


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("branch", [False, True])
def test_a_given_dx_is_written_without_norm(dtype, branch):
    dy = torch.randn(3, 5, 36, device="cuda").to(dtype)
    h = torch.randn_like(dy) if branch else None
    dx = torch.full_like(dy, 7.0)
    got = quan.residual_join_backward(dy, None, None, h, dx=dx)
    assert got[0] is dx and torch.equal(dx, dy)
    assert (got[1] is not None) == branch
    assert quan.residual_join_backward(dy, None, None, h)[0] is dy
    for bad in (dict(dn=dy), dict(dn=None, dh=dx) if not branch else dict(dn=dy)):
        with pytest.raises(quan.QuanError):
            quan.residual_join_backward(dy, y=None, h=h, **bad)
