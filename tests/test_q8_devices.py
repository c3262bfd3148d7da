"""Where the 8-bit operators' operands live (no device needed: the library is a stand-in that records calls)."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2406_20037_amd import _lib as L  # noqa: E402


class On:
    """A tensor as the binding looks at it, on the given GPU."""

    def __init__(self, t, device):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index


def matrix(rows, cols, device=-1):
    m = L.Q8(rows, cols, device="cpu")
    m._device = device
    return m


def calls(on=-1):
    """Each entry point with every operand on one device."""
    x = On(torch.zeros(4, 256), on)
    m, m_t, wide, wide_t = (matrix(r, c, on) for r, c in ((4, 256), (256, 4), (4, 512), (512, 4)))
    return [lambda s=None, x=x, m=m, t=m_t: L.ds_q8_quantize(x, m, t, stream=s),
            lambda s=None, x=x, m=m, t=None: L.ds_q8_matmul(m, matrix(256, 256, on), x, stream=s),
            lambda s=None, x=On(torch.zeros(4, 512), on), m=m, t=wide: L.ds_swiglu8(x, m, t, stream=s),
            lambda s=None, x=x, m=wide, t=wide_t: L.ds_swiglu8_grad(m, x, wide, t, m_t, stream=s)]


@pytest.fixture
def launched(monkeypatch):
    """(entry point, current GPU, stream) of each call of the library."""
    at, seen = [0], []

    class Device:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            self.was, at[0] = at[0], self.d

        def __exit__(self, *_):
            at[0] = self.was

    names = ("ds_q8_quantize", "ds_q8_matmul", "ds_swiglu8", "ds_swiglu8_grad")
    monkeypatch.setattr(L, "lib", types.SimpleNamespace(
        **{n: lambda *a, n=n: seen.append((n, at[0], a[-1])) or L.DS_OK for n in names}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(L, "_raw_stream", lambda d: 1000 + d)
    return seen


def test_host_memory_is_refused(launched):
    for call in calls():
        with pytest.raises(ValueError, match="the host"):
            call()
    assert not launched


def test_two_devices_are_refused(launched):
    for call in calls(0):
        for wrong in (-1, 1):
            for name, m in zip("mt", call.__defaults__[2:]):
                if m is not None:
                    with pytest.raises(ValueError, match="not on one GPU"):
                        call(**{name: matrix(m.rows, m.cols, wrong)})
    assert not launched


@pytest.mark.parametrize("device", [0, 1])
def test_the_operands_device_and_its_stream(launched, device):
    for call in calls(device):
        call()
    assert [(d, s) for _, d, s in launched] == [(device, 1000 + device)] * 4
    assert torch.cuda.current_device() == 0


def test_a_stream_of_another_device_is_refused(launched):
    for call in calls(1):
        call(s=types.SimpleNamespace(device_index=1, cuda_stream=77))
        with pytest.raises(ValueError, match="stream"):
            call(s=types.SimpleNamespace(device_index=0, cuda_stream=78))
    assert [s for _, _, s in launched] == [77] * 4
