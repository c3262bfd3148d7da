"""What the 8-bit layer keeps from pass to pass (no device: the operators are stand-ins that do nothing)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2406_20037_amd import mlp8  # noqa: E402


@pytest.fixture
def layer(monkeypatch):
    for name in ("ds_q8_quantize", "ds_q8_matmul", "ds_swiglu8", "ds_swiglu8_grad"):
        monkeypatch.setattr(mlp8.L, name, lambda *a, **k: None)
    return mlp8.Mlp8(32, 48, device="cpu")


def kept(layer):
    return sum(len(sets) for sets in layer._buffers.values())


def test_many_token_counts_keep_few_sets(layer):
    for n in range(1, 60):
        layer.forward(torch.zeros(n, 32), train=n % 3 == 0)
    assert kept(layer) == 2 * mlp8.SETS


def test_a_set_serves_the_next_pass(layer):
    y = layer.forward(torch.zeros(7, 32))
    for n in (1, 2, 7, 3):
        layer.forward(torch.zeros(n, 32))
    assert layer.forward(torch.zeros(7, 32)) is y and kept(layer) == 4
    for n in (10, 11, 12):
        layer.forward(torch.zeros(n, 32))
    assert layer.forward(torch.zeros(7, 32)) is y


def test_answers_between_do_not_take_what_backward_needs(layer):
    layer.forward(torch.zeros(7, 32), train=True)
    held = layer._buffers[True][7]["saved"]
    for n in range(1, 20):
        layer.forward(torch.zeros(n, 32))
    dx, dw1, dw2 = layer.backward(torch.zeros(7, 32))
    assert layer._buffers[True][7]["saved"] is held and dx.shape == (7, 32) and dw2.shape == (32, 48)


def test_backward_without_its_forward_is_refused(layer):
    layer.forward(torch.zeros(7, 32), train=True)
    layer.forward(torch.zeros(5, 32))
    for n in (5, 6):
        with pytest.raises(ValueError, match=f"{n} tokens"):
            layer.backward(torch.zeros(n, 32))
