"""The residual block's Python helpers without a GPU: what they hand to the library, seen through
stand-ins for CUDA tensors and for the packed call."""
import struct

import pytest

torch = pytest.importorskip("torch")

from paper_2509_05512_gb300 import build, quan


class Device:
    """A CUDA tensor's face: what the helpers look at, and an address that is never read."""

    def __init__(self, shape, dtype, *, at=0x10000000, cuda=0, contiguous=True):
        self.shape, self.dtype = torch.Size(shape), dtype
        self.device = torch.device("cuda", cuda) if cuda >= 0 else torch.device("cpu")
        self.is_cuda = cuda >= 0
        self._at, self._contiguous = at, contiguous

    def data_ptr(self):
        return self._at

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def is_contiguous(self):
        return self._contiguous

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def reshape(self, *shape):
        return self


@pytest.fixture
def calls(monkeypatch):
    """The packed calls made, as (entry point number, words); allocations are stand-ins."""
    build.build_library()
    quan.load()
    made, at = [], iter(range(0x70000000000, 1 << 60, 1 << 34))
    monkeypatch.setattr(quan, "_call", lambda op, words: made.append(
        (op, struct.unpack("%dq" % (len(words) // 8), words))))
    monkeypatch.setattr(quan, "_stream", lambda *a: 0)
    monkeypatch.setattr(quan, "_empty", lambda stream, shape, dtype, device: Device(
        (shape,) if isinstance(shape, int) else shape, dtype, at=next(at)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return made


F32, BF16 = torch.float32, torch.bfloat16


def test_a_given_dx_is_written_without_norm_and_branch(calls):
    # the join without pre-norm and branch has dx = dy: a buffer for dx must be filled all the same
    dy = Device((2, 3, 64), F32, at=0x20000000)
    dx = Device((2, 3, 64), F32, at=0x30000000)
    assert quan.residual_join_backward(dy, None, None)[0] is dy and not calls
    got = quan.residual_join_backward(dy, None, None, dx=dx)
    assert got[0] is dx and got[1:] == (None,) * 4
    (op, words), = calls
    assert op == 15 and words[0] == 0x20000000 and words[-6] == 0x30000000


@pytest.mark.parametrize("extra", ["dn", "dh"])
def test_a_gradient_that_belongs_to_nothing_reaches_the_checks(calls, extra):
    # dn without pre, dh without h: the library refuses them, the helper may not drop them
    dy, t = (Device((2, 3, 64), F32, at=a) for a in (0x20000000, 0x30000000))
    args = {"dn": None, "y": None, extra: t}
    quan.residual_join_backward(dy, **args)
    (op, words), = calls
    assert op == 15 and 0x30000000 in words


def letters(Cin, Cout, transposed=False, **kw):
    n, k = (Cin // 4, Cout // 4) if transposed else (Cout // 4, Cin // 4)
    q = dict(dict(shape=(4, n, (k + 15) // 16 * 16), dtype=torch.float8_e4m3fn, at=0x40000000),
             **kw.get("q", {}))
    s = dict(dict(shape=(4, -(-n // 128), -(-k // 128)), dtype=F32, at=0x50000000),
             **kw.get("scale", {}))
    return quan.F8Weights(Device(**q), Device(**s), Cin, Cout, transposed)


def product(x=None, w=None, **kw):
    return quan.qpointwise_f8(x or Device((1000, 64), BF16), w or letters(64, 128), **kw)


def gradient(x=None, w=None, **kw):
    return quan.qpointwise_f8_backward_data(x or Device((1000, 128), BF16),
                                            w or letters(64, 128, True), **kw)


def join_gradient(**kw):
    t = [Device((1000, 64), F32, at=0x20000000 + (k << 24)) for k in range(4)]
    v = Device((64,), F32, at=0x1000000)
    return quan.residual_join_backward(*t, pre=v, **kw)


BAD_WORKSPACES = [dict(cuda=-1), dict(contiguous=False)]


@pytest.mark.parametrize("call", [product, gradient, join_gradient])
def test_workspaces_are_looked_at(calls, call):
    # the library gets an address and a byte count: one on the host faults, and a strided view is
    # written past its elements
    good = Device((1 << 20,), torch.uint8, at=0x60000000)
    call(workspace=good)
    (_, words), = calls
    assert 0x60000000 in words and 1 << 20 in words
    for bad in BAD_WORKSPACES:
        with pytest.raises(ValueError, match="workspace must be a contiguous CUDA tensor"):
            call(workspace=Device((1 << 20,), torch.uint8, **bad))
    assert len(calls) == 1


BAD_LETTERS = [
    ("q", dict(cuda=-1)), ("q", dict(contiguous=False)), ("q", dict(dtype=torch.uint8)),
    ("q", dict(shape=(4, 32, 15))), ("q", dict(shape=(4, 16, 16))), ("q", dict(shape=(0,))),
    ("scale", dict(cuda=-1)), ("scale", dict(contiguous=False)), ("scale", dict(dtype=BF16)),
    ("scale", dict(shape=(3, 1, 1))),
    ("scale", dict(shape=(0,))),
]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("part, bad", BAD_LETTERS)
def test_letters_are_looked_at(calls, part, bad, transposed):
    # F8Weights is a tuple that anyone can put together; the kernels read as much of it as the
    # channel counts say
    call = gradient if transposed else product
    call(w=letters(64, 128, transposed))
    with pytest.raises(ValueError, match="w.%s must be a contiguous CUDA tensor" % part):
        call(w=letters(64, 128, transposed, **{part: bad}))
    assert len(calls) == 1


def test_channel_counts_that_the_letters_do_not_have(calls):
    # all that fits 64 -> 128 but not the counts beside it
    w = letters(64, 128)
    with pytest.raises(ValueError, match="w.q"):
        product(w=w._replace(Cout=256))
    with pytest.raises(ValueError, match="w.q"):
        product(x=Device((1000, 2048), BF16), w=w._replace(Cin=2048))
    # 130 output channels a component need a second row of scales
    w = letters(64, 520)
    with pytest.raises(ValueError, match="w.scale"):
        product(w=w._replace(scale=letters(64, 128).scale))
    assert not calls


def test_tensors_of_another_device_are_refused(calls, monkeypatch):
    # a launch goes to the current device, where another one's memory need not be mapped
    here = dict(x=Device((1000, 64), BF16), w=letters(64, 128))
    there = Device((128,), F32, cuda=1)
    with pytest.raises(ValueError, match="bias"):
        product(**here, bias=there)
    with pytest.raises(ValueError, match="w.q"):
        product(w=letters(64, 128, q=dict(cuda=1)))
    with pytest.raises(ValueError, match="w.scale"):
        gradient(w=letters(64, 128, True, scale=dict(cuda=1)))
    with pytest.raises(ValueError, match="workspace"):
        product(**here, workspace=Device((1 << 20,), torch.uint8, cuda=1))
    with pytest.raises(ValueError, match="out"):
        product(**here, out=Device((1000, 128), BF16, cuda=1))
    x, v = Device((1000, 64), F32), Device((64,), F32)
    far = Device((1000, 64), F32, cuda=1)
    for bad in (dict(h=far), dict(h=x, y=far), dict(pre=Device((64,), F32, cuda=1)),
                dict(pre=v, n=far), dict(h=x, post=Device((64,), F32, cuda=1)),
                dict(h=x, gate=Device((64,), F32, cuda=1)),
                dict(h=x, counter=Device((1,), torch.int64, cuda=1))):
        with pytest.raises(ValueError, match="must be a contiguous CUDA tensor"):
            quan.residual_join(x, **bad)
    for bad in (dict(dn=far), dict(y=far), dict(h=far), dict(dx=far), dict(h=x, dh=far)):
        with pytest.raises(ValueError, match="must be a contiguous CUDA tensor"):
            quan.residual_join_backward(x, **dict(dict(dn=x, y=x, pre=v), **bad))
    with pytest.raises(ValueError, match="out"):
        quan.dropout(x, 0.5, 1, out=far)
    w = [Device((32, 1, 1, 16), BF16, cuda=int(k == 2)) for k in range(4)]
    with pytest.raises(ValueError, match="wj"):
        quan.quantize_f8_weights(*w)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: product(**here), lambda: gradient(), lambda: quan.residual_join(x, pre=v),
                 lambda: quan.residual_join_backward(x, x, x, pre=v),
                 lambda: quan.dropout(x, 0.5, 1), lambda: quan.quantize_f8_weights(*w)):
        with pytest.raises(ValueError, match="current device is cuda:1"):
            call()
    assert not calls


def test_sizes_past_32_bits_are_not_cut():
    # the packed entry takes 64-bit words: a size that the C function's int does not hold is refused,
    # not taken modulo 2^32.  Without rows nothing would be launched.
    build.build_library()
    quan.load()
    for C in ((1 << 32) + 64, (1 << 32), -(1 << 32) + 64, 1 << 62):
        with pytest.raises(quan.QuanError):
            quan.quan_residual_join_fwd(None, None, None, None, None, 0, C, 4, 1, 0, 1.0, 1e-5, 0.0,
                                        1, 0, None, None, None, 0)
        with pytest.raises(quan.QuanError):
            quan.quan_residual_join_bwd(None, None, None, None, None, None, None, 0, C, 4, 1, 0,
                                        1.0, 1e-5, 0.0, 1, 0, None, None, 0, None, None, None, None,
                                        None, 0)
        with pytest.raises(quan.QuanError):
            quan.quan_qpoint_f8_fwd(None, None, None, None, None, None, 0, C, 64, 0, None, 0, None,
                                    0)
        with pytest.raises(quan.QuanError):
            quan.quan_qpoint_f8_bwd_data(None, None, None, 0, 64, C, None, 0, None, 0)


def test_letters_past_32_bits_are_refused(calls, monkeypatch):
    made = []
    monkeypatch.setattr(quan, "quan_f8_weights", lambda *a: made.append(a))
    w = [Device((16, 1, 1, (1 << 30) + 16), BF16) for _ in range(4)]  # Cin = 2^32 + 64
    for transpose in (False, True):
        with pytest.raises(ValueError, match="channels"):
            quan.quantize_f8_weights(*w, transpose=transpose)
    quan.quantize_f8_weights(*[Device((16, 1, 1, 16), BF16) for _ in range(4)])
    assert len(made) == 1


def test_addresses_of_integer_types():
    # what the raw functions take for a tensor: an address of int or a type derived from it
    class Address(int):
        pass

    assert quan._addr(Address(0x1000)) == 0x1000 and quan._addr(0x1000) == 0x1000
    assert quan._addr(Device((1,), F32, at=0x2000)) == 0x2000 and quan._addr(None) == 0
    with pytest.raises(AttributeError):
        quan._addr("x")
