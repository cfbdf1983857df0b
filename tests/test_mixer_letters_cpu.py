"""Which letters the mixing stack's quantised forms stand for, with the quantisers replaced by ones
that keep what they were given."""
import pytest

torch = pytest.importorskip("torch")

from paper_2509_05512_gb300 import mixer, quan


@pytest.fixture
def model(monkeypatch):
    keep = lambda *w, **_: tuple(x.clone() for x in w)
    for name in ("quantize_f8_weights", "quantize_w4_weights"):
        monkeypatch.setattr(quan, name, keep)
    monkeypatch.setattr(quan, "residual_join", lambda x, h=None, **_: (x, x))
    monkeypatch.setattr(quan, "qpointwise_w4", lambda x, w: served.append(w) or x)
    served.clear()
    return mixer.Mixer(16, 2, device="cpu")


served = []


def gradients(m):
    one = lambda v: [torch.ones_like(t) for t in v]
    return {"letters": [[torch.ones(w.shape) for w in l] for l in m.letters],
            "pre": one(m.pre), "post": one(m.post), "gate": one(m.gate)}


def test_letters_served_are_those_of_the_last_update(model):
    x = torch.zeros(1, 16, dtype=torch.bfloat16)
    model.quantize_4bit()
    model.serve(x)
    assert all(torch.equal(a, b) for s, l in zip(served, model.letters) for a, b in zip(s, l))
    model.update(gradients(model), 0.5)
    served.clear()
    with pytest.raises(RuntimeError, match="quantize_4bit"):
        model.serve(x)  # (the letters in 4 bits are those of before the update)
    assert not served
    model.quantize_4bit()
    model.serve(x)
    assert len(served) == 2
    assert all(torch.equal(a, b) for s, l in zip(served, model.letters) for a, b in zip(s, l))


def test_an_update_leaves_what_a_captured_pass_reads(model):
    # a graph of serve holds the letters' addresses: the tensors stay until quantize_4bit makes others
    model.quantize_4bit()
    before = model.w4
    model.update(gradients(model), 0.5)
    assert model.w4 is before


def test_letters_have_to_be_quantised_before_they_are_served(model):
    with pytest.raises(RuntimeError, match="quantize_4bit"):
        model.serve(torch.zeros(1, 16, dtype=torch.bfloat16))
    model.quantize_4bit()
    model.letters[0][0].zero_()  # changed by hand, and said so
    model.quantize()
    with pytest.raises(RuntimeError, match="quantize_4bit"):
        model.serve(torch.zeros(1, 16, dtype=torch.bfloat16))
