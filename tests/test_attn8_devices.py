"""Where the operands of the operators around attention live (no device needed: the library is a stand-in that
records calls)."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2406_20037_amd import _lib as L  # noqa: E402
from test_q8_devices import On  # noqa: E402


class Device:
    at = 0

    def __init__(self, d):
        self.d = d

    def __enter__(self):
        self.was, Device.at = Device.at, self.d

    def __exit__(self, *_):
        Device.at = self.was


def calls(on):
    """Each entry point with its operands, all on one device: name, call(operands, stream), operands."""
    def heads(h):
        return On(torch.zeros(3, h, 32), on)

    def held(thing):
        thing._device = on
        return thing
    lists = [torch.zeros(n, dtype=torch.int32) for n in (3, 2)] + [torch.zeros(2, 4, dtype=torch.int32)]
    cache, chunk = held(L.Cache8(5, 2, 32, 16, device="cpu")), held(L.Chunk(*lists))
    pos, freqs = On(torch.zeros(3, dtype=torch.int32), on), On(torch.zeros(16), on)
    rows = dict(cache=cache, chunk=chunk, k=heads(2), v=heads(2))
    return [("ds_rotary", lambda o, s=None: L.ds_rotary(o["x"], o["pos"], o["freqs"], o["y"], stream=s),
             dict(x=heads(4), pos=pos, freqs=freqs, y=heads(4))),
            ("ds_cache8_write", lambda o, s=None: L.ds_cache8_write(o["cache"], o["chunk"], o["k"], o["v"], s), rows),
            ("ds_cache8_read", lambda o, s=None: L.ds_cache8_read(o["cache"], o["chunk"], o["k"], o["v"], s), rows),
            ("ds_attn8", lambda o, s=None: L.ds_attn8(o["q"], o["cache"], o["chunk"], o["out"], o["lse"], work=o["work"], stream=s),
             dict(q=heads(4), cache=cache, chunk=chunk, out=heads(4), lse=On(torch.zeros(3, 4), on),
                  work=On(torch.zeros(16, dtype=torch.uint8), on)))]


@pytest.fixture
def launched(monkeypatch):
    seen = []
    names = ("ds_rotary", "ds_cache8_write", "ds_cache8_read", "ds_attn8")
    monkeypatch.setattr(Device, "at", 0)
    monkeypatch.setattr(L, "lib", types.SimpleNamespace(
        **{n: lambda *a, n=n: seen.append((n, Device.at, a[-1])) or L.DS_OK for n in names}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: Device.at)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(L, "_raw_stream", lambda d: 1000 + d)
    monkeypatch.setattr(L, "ptr", lambda t: t and t.data_ptr())
    return seen


def test_operands_apart_are_refused(launched):
    for _, call, operands in calls(0):
        for name, thing in operands.items():
            for wrong in (-1, 1):
                if isinstance(thing, On):
                    other = On(thing.t, wrong)
                else:
                    other = types.SimpleNamespace(**{**vars(thing), "_device": wrong})
                with pytest.raises(ValueError, match="not on one GPU"):
                    call({**operands, name: other})
    for _, call, operands in calls(-1):
        with pytest.raises(ValueError, match="the host"):
            call(operands)
    assert not launched


@pytest.mark.parametrize("device", [0, 1])
def test_the_operands_device_and_its_stream(launched, device):
    names = [name for name, call, operands in calls(device) if call(operands) is not False]
    assert launched == [(name, device, 1000 + device) for name in names]
    assert Device.at == 0


def test_a_stream_of_another_device_is_refused(launched):
    for name, call, operands in calls(1):
        call(operands, types.SimpleNamespace(device_index=1, cuda_stream=77))
        with pytest.raises(ValueError, match="stream"):
            call(operands, types.SimpleNamespace(device_index=0, cuda_stream=78))
    assert [s for _, _, s in launched] == [77] * 4


def test_lists_on_two_devices_are_refused():
    a, b, c = (On(torch.zeros(*n, dtype=torch.int32), d) for n, d in (((3,), 0), ((2,), 0), ((2, 4), 1)))
    with pytest.raises(ValueError, match="one device"):
        L.Chunk(a, b, c)
    k = On(torch.zeros(2, 1, 16, 16, dtype=torch.uint8).view(torch.float8_e4m3fn), 0)
    s = On(torch.zeros(2, 1, 16), 1)
    with pytest.raises(ValueError, match="one device"):
        L.Cache8.of(k, k, s, s)
