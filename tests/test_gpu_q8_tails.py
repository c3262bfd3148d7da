"""The gated unit at gates far from 0, where sigmoid is 0 or 1 to fp32: silu(g) goes to 0 or g however large
|g| is.  Bounds: 2^-20 of the value for fp32's roundings, and for values beside 0 what fp32 has no normal number
for, times the other factor."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_q8 import check_q8, env, make, typed  # noqa: F401

pytestmark = pytest.mark.gpu

GATES = [-3e38, -1e38, -1e30, -1e15, -1e6, -1e4, -1000.0, -200.0, -120.0, -104.0, -90.0, -88.6, -88.5, -88.0,
         -87.4, -87.0, -60.0, -17.0, 17.0, 60.0, 87.0, 88.5, 88.6, 104.0, 1e4, 1e15, 1e30]


def rows(cols):
    """A row a gate, the other factor from -2 to 2."""
    g = np.repeat(np.array(GATES)[:, None], cols, 1)
    return g, np.repeat(np.linspace(-2, 2, cols)[None], len(GATES), 0)


def silu(g):
    """g / (1 + exp(-g)) in 64 bits, whose exp is infinite from 710 on, which gives 0 as it should."""
    return g * q8.sigmoid(g)


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
def test_forward(env, name, kind):  # noqa: F811
    torch, L = env
    g, u = rows(128)
    gu, e = typed(torch, np.concatenate([g, u], 1), name)
    g, u = e[:, :128], e[:, 128:]
    h = make(torch, L, len(GATES), 128, q8.E4M3, kind)
    L.ds_swiglu8(gu, h)
    torch.cuda.synchronize()
    want = silu(g) * u
    check_q8(h, want, q8.E4M3, kind, noise=2.0 ** -20 * np.abs(want) + 2.0 ** -126 * 90 * (1 + np.abs(u)))


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("whole", [False, True])
def test_gradient(env, name, whole):  # noqa: F811
    torch, L = env
    cols = 128
    g, u = rows(cols)
    if whole:                                          # as many rows as a tile
        g, u = np.resize(g, (128, cols)), np.resize(u, (128, cols))
    n = len(g)
    # one scale a row: gates of +-448 or so times it
    saved = make(torch, L, n, 2 * cols, q8.E4M3, q8.F32)
    x, _ = typed(torch, np.concatenate([g, u], 1), "float32")
    L.ds_q8_quantize(x, saved, None)
    torch.cuda.synchronize()
    v = saved.values().double().cpu().numpy()
    g, u = v[:, :cols], v[:, cols:]
    dh, d = typed(torch, np.repeat(np.linspace(-1, 1, n)[:, None], cols, 1), name)
    s = q8.sigmoid(g)
    slope = s * (1 + g * (1 - s))
    tiny = 2.0 ** -126 * 90 * (1 + np.abs(d)) * (1 + np.abs(u))
    want = np.concatenate([d * u * slope, d * silu(g)], 1)
    # 1 + g (1 - s) passes 0, so its rounding is relative to 1 + |g| (1 - s); and 1 - s is off by up to 2^-22,
    # from g = 32 on by nothing (1 + exp(-g) is 1 in fp32)
    off = 2.0 ** -20 * (1 + np.abs(g) * (1 - s)) + 2.0 ** -22 * np.minimum(np.abs(g), 32.0)
    noise = np.concatenate([np.abs(d * u) * s * off, 2.0 ** -20 * np.abs(d * silu(g))], 1) + \
        np.concatenate([tiny, tiny], 1)
    h = silu(g) * u
    for fmt in (q8.E4M3, q8.E5M2):
        out = [make(torch, L, n, 2 * cols, fmt, q8.F32), make(torch, L, 2 * cols, n, fmt, q8.F32),
               make(torch, L, cols, n, q8.E4M3, q8.F32)]
        L.ds_swiglu8_grad(saved, dh, *out)
        torch.cuda.synchronize()
        check_q8(out[0], want, fmt, q8.F32, noise=noise)
        check_q8(out[1], want.T, fmt, q8.F32, noise=noise.T)
        check_q8(out[2], h.T, q8.E4M3, q8.F32, noise=(2.0 ** -20 * np.abs(h) + tiny).T)
