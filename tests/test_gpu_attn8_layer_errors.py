"""The attention layer after a call that raised part of the way: as if it had not been made."""
import pytest

from test_gpu_attn8_layer import make
from test_gpu_cache8 import env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["ds_rotary", "ds_cache8_write", "ds_attn8", "ds_q8_matmul"])
def test_a_call_that_raises(env, name, monkeypatch):  # noqa: F811
    torch, L = env
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = [torch.randn(sum(n), 128, generator=gen, device="cuda", dtype=torch.bfloat16) for n in ([30, 0, 7], [2, 20, 1])]
    other = torch.randn(44, 128, generator=gen, device="cuda", dtype=torch.bfloat16)
    layer, straight = make(), make()

    def broken(*args, **kw):
        raise RuntimeError("no memory")
    layer.forward(x[0], [30, 0, 7])
    before = (layer.lengths[:], layer.free[:], [h[:] for h in layer.held])
    with monkeypatch.context() as m:
        inner = getattr(L, name)
        # (the last product, not the first)
        m.setattr(L, name, broken if name != "ds_q8_matmul" else lambda a, b, c, **kw: broken() if b is layer.qo else inner(a, b, c, **kw))
        with pytest.raises(RuntimeError, match="no memory"):
            layer.forward(other, [4, 39, 1])
    assert (layer.lengths, layer.free, layer.held) == before
    straight.forward(x[0], [30, 0, 7])
    assert torch.equal(layer.forward(x[1], [2, 20, 1]), straight.forward(x[1], [2, 20, 1]))
    torch.cuda.synchronize()


def test_turned_values_past_a_head(env):  # noqa: F811
    torch, L = env
    for kw in (dict(turn=64), dict(turn=None, freqs=torch.ones(25))):
        with pytest.raises(ValueError, match="turned"):
            make(**kw)
