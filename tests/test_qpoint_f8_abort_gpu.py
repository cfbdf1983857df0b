"""The 8-bit product gives up in an orderly way: a barrier that nothing arrives on ends the call with
a status after the limit, every copy and product under way is waited for, and the next call is
right.  Rows and channels such that the copies all fit the ring, or do not, and one or several
tiles a CTA."""
import pytest

torch = pytest.importorskip("torch")

from paper_2509_05512_gb300 import build, quan

pytestmark = pytest.mark.gpu

DRAIN = 8  # the status bit of a drain that ran out of time


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    quan.load()
    yield
    assert quan.quan_device_status()[0] == quan.QUAN_OK


@pytest.mark.parametrize("act", [quan.QUAN_ACT_NONE, quan.QUAN_ACT_SILU])
@pytest.mark.parametrize("rows, Cin, Cout", [(100, 256, 512), (300, 2048, 512), (3000, 1028, 1024),
                                             (20000, 512, 256)])
def test_an_abort_ends_in_order(rows, Cin, Cout, act):
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = [(torch.randn(Cout // 4, 1, 1, Cin // 4, generator=g, device="cuda") / Cin ** 0.5)
         .to(torch.bfloat16) for _ in range(4)]
    x = torch.randn(rows, Cin, generator=g, device="cuda").to(torch.bfloat16)
    f = quan.quantize_f8_weights(*w)
    want = quan.qpointwise_f8(x, f, act=act)
    assert quan.quan_device_status()[0] == quan.QUAN_OK
    quan.quan_set_wait_limit_ns(20_000_000)
    quan.quan_set_fault_injection(True)
    try:
        quan.qpointwise_f8(x, f, act=act)
        status, bits = quan.quan_device_status()
    finally:
        quan.quan_set_fault_injection(False)
        quan.quan_set_wait_limit_ns(0)
    assert status == quan.QUAN_ERR_DEVICE_TIMEOUT and bits and not bits & DRAIN
    for _ in range(2):
        assert torch.equal(quan.qpointwise_f8(x, f, act=act), want)
