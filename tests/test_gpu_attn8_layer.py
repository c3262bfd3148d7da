"""The attention layer: prompts at once, in chunks and token by token give the same as its own operators one by one,
and as the oracle's attention over what its cache holds."""
import json

import numpy as np
import pytest

from oracle import attn8 as oracle
from test_gpu_cache8 import HALF, env  # noqa: F401

pytestmark = pytest.mark.gpu


def make(**kw):
    from paper_2406_20037_amd.attn8 import Attention8
    return Attention8(128, 4, 2, 48, **{**dict(seqs=3, most=200, page=16, turn=32, seed=3), **kw})


def test_chunks_and_tokens(env):  # noqa: F811
    """Rows that pass through products of many rows are the same bits in the cache however the prompt is cut.  A product
    of few rows (the last chunk's two) adds its fp32 sums in another order, so that a projected value x may
    round to bf16 the other way: it is off by 2^-7 |x|, and by twice the sums' own error d, 2^-24 * 128 of
    the sum of magnitudes (some 8, for values of 1 in rows whose largest M is over 1: d < 2^-13 M).  Turning takes pairs, whose
    length is at most sqrt(2) M, so a turned value is off by sqrt(2) (2^-7 M + d), and by 2^-7 M for its
    own rounding: less than 2^-5 M together.  Either side then rounds to e4m3 by 2^-4 of itself (below the normal ones by 2^-10 of a scale
    of at most M / 224): 2^-3 of the larger one + 2^-5 M.

    Outputs of attention differ by the roundings of weights and of themselves to bf16, on either side, about 2^-8 of
    their size in the mean.  A value that far off rounds to the other side of a step of e4m3, 2^-3 to 2^-4 of it, with a
    probability of the difference over the step, so the mean square of the difference is
    (2^-8)(2^-3.5) of the value's: a root of 2^-5.75, which the product with independent weights keeps.  2^-4 is
    three times that."""
    torch, L = env
    gen = torch.Generator(device="cuda").manual_seed(4)
    lens = [120, 33, 1]
    x = [torch.randn(n, 128, generator=gen, device="cuda", dtype=torch.bfloat16) for n in lens]
    cut_last = [1, 0, 1]
    for window in (0, 40):
        whole = make(window=window)
        want = whole.forward(torch.cat(x), lens).split(lens)
        cut = make(window=window)
        parts = [[], [], []]
        at = [0, 0, 0]
        for new in ([50, 33, 0], [69, 0, 0], cut_last):
            y = cut.forward(torch.cat([x[s][at[s]:at[s] + n] for s, n in enumerate(new)]), new).split(new)
            for s, n in enumerate(new):
                parts[s].append(y[s])
                at[s] += n
        torch.cuda.synchronize()
        for s in range(3):
            a = [t[:, :, :].float() for t in (whole.cache.values()[0][whole.table[s].long().cuda()],
                                              cut.cache.values()[0][cut.table[s].long().cuda()])]
            rows = lens[s]
            a = [t.transpose(1, 2).flatten(0, 1)[:rows] for t in a]
            many = rows - cut_last[s]
            assert torch.equal(a[0][:many], a[1][:many]), s
            top = a[0].abs().amax(-1, keepdim=True)
            assert bool(((a[0] - a[1]).abs() <= 2.0 ** -3 * torch.maximum(a[0].abs(), a[1].abs()) + 2.0 ** -5 * top).all()), s
            got = torch.cat(parts[s]).float()
            assert float((got - want[s].float()).norm() / want[s].float().norm()) < 2.0 ** -4


def test_against_the_oracle(env):  # noqa: F811
    """The attention inside, from the layer's own queries."""
    torch, L = env
    layer = make(pairs=True)
    seen = []
    inner = L.ds_attn8

    def watch(q, cache, chunk, out, **kw):
        r = inner(q, cache, chunk, out, **kw)
        seen.append((q, out, kw))
        return r
    L.ds_attn8 = watch
    try:
        gen = torch.Generator(device="cuda").manual_seed(5)
        for new in ([30, 0, 7], [2, 5, 1]):
            layer.forward(torch.randn(sum(new), 128, generator=gen, device="cuda", dtype=torch.bfloat16), new)
    finally:
        L.ds_attn8 = inner
    torch.cuda.synchronize()
    k, v = (t.double().cpu().numpy() for t in layer.cache.values())
    table = layer.table.numpy()
    q, out, _ = seen[-1]
    t = 0
    for s, n in enumerate([2, 5, 1]):
        length = layer.lengths[s]
        j = np.arange(length)
        kb, vb = (m[table[s, j // 16], :, j % 16] for m in (k, v))
        for i in range(n):
            for h in range(4):
                row, _, room, _ = oracle.attend(q[t, h].double().cpu().numpy(), kb[:, h // 2], vb[:, h // 2],
                                                j <= length - n + i, 48 ** -0.5)
                # a weight's rounding (2^-8) and all fp32 ones (2^-12 over 40 keys of 48 values), then the output's
                lim = room * (2.0 ** -8 + 2.0 ** -12) + np.abs(row) * HALF["bfloat16"]
                assert (np.abs(out[t, h].double().cpu().numpy() - row) <= lim * 1.01).all()
            t += 1


def test_pages_and_refusals(env):  # noqa: F811
    torch, L = env
    layer = make(most=40)
    x = torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16)
    for bad in ([1, 1], [5, -1, 0], [4, 0, 1]):
        with pytest.raises(ValueError):
            layer.forward(x, bad)
    with pytest.raises(ValueError, match="tokens"):
        layer.forward(torch.zeros(49, 128, device="cuda", dtype=torch.bfloat16), [49, 0, 0])
    assert layer.lengths == [0, 0, 0] and len(layer.free) == 9
    layer.forward(torch.zeros(57, 128, device="cuda", dtype=torch.bfloat16), [17, 40, 0])
    assert [len(h) for h in layer.held] == [2, 3, 0] and len(set(sum(layer.held, []) + layer.free)) == 9
    layer.forget(1)
    assert len(layer.free) == 7 and layer.lengths[1] == 0
    y = layer.forward(torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16), [1, 2, 1])
    torch.cuda.synchronize()
    assert torch.isfinite(y).all()
    assert layer.forward(x[:0], [0, 0, 0]).shape == (0, 128)


def test_command(env, capsys):  # noqa: F811
    from paper_2406_20037_amd import attn8
    attn8.main(["--width", "128", "--heads", "4", "--kv-heads", "2", "--dim", "32", "--prompt", "70", "--chunk", "32",
                "--tokens", "3", "--seqs", "2"])
    line = json.loads(capsys.readouterr().out)
    assert line["finite"] and line["chunks_off"] < 2.0 ** -4


def test_long_text_frequencies():
    import torch
    from paper_2406_20037_amd.attn8 import rotary_freqs
    f = rotary_freqs(64)
    assert f.shape == (32,) and float(f[0]) == 1.0 and torch.allclose(rotary_freqs(64, factor=4.0), f / 4)
    g = rotary_freqs(64, factor=8.0, trained=4096)
    turns = 4096 * f.double() / (2 * np.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 8)
    assert bool((g <= f).all()) and bool((g >= f / 8 * (1 - 1e-6)).all())
