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


def owner(t):
    """The stream that the allocator keeps t's memory for."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not an allocation of torch's")


def test_what_a_helper_allocates_belongs_to_its_stream():
    # memory that belongs to another stream would be handed on while the call still uses it;
    # the handle 0 is the default stream, whatever stream is current
    x = torch.randn(1 << 22, device="cuda")  # its result is an allocation of its own
    side = torch.cuda.Stream()
    default = torch.cuda.default_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for stream, handle in ((None, side.cuda_stream), (side, side.cuda_stream),
                               (side.cuda_stream, side.cuda_stream), (default, 0), (0, 0)):
            assert owner(quan.dropout(x, 0.5, 1, stream=stream)) == handle
    torch.cuda.synchronize()
