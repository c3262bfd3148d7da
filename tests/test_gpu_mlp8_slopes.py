"""The 8-bit layer's three gradients along directions in x, w1 and w2 against the loss's slope in 64 bits.

Along one direction roundings average out, so the bound is far below the gradients' own 10%.  It is six
standard deviations of what the layer's roundings do to the slope: each value that is rounded is off by a
relative amount of its own, 2.6% of it in the mean square in e4m3 and 5.2% in e5m2 (bf16's 2^-9 is beside that), and
the slope's derivatives with respect to all of these amounts are taken in 64 bits.  Two roundings of one value,
along rows and along columns, are the same with power-of-two scales and apart with others: the larger of the two sums
counts.  Beyond first order the bound allows the square of the relative amounts, 0.3%, of all terms' magnitudes.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E4M3, E5M2 = 0.026, 0.052


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a device"
    from paper_2406_20037_amd import mlp8
    return torch, mlp8


def loss(torch, x, w1, w2, dy, hidden, up):
    gu = x @ w1.t()
    h = torch.nn.functional.silu(gu[:, :hidden]) * gu[:, up:]
    return ((h @ w2.t()) * dy).sum()


def gradients(torch, x, w1, w2, dy, hidden, up, e):
    """(dx, dw1, dw2) by the layer's own steps, each rounded value v as v (1 + e)."""
    gu = (x * (1 + e["x"])) @ (w1 * (1 + e["w1"])).t()
    kept = gu * (1 + e["kept"])
    g, u = kept[:, :hidden], kept[:, up:]
    s = torch.sigmoid(g)
    dh = (dy * (1 + e["dy"])) @ (w2 * (1 + e["w2"]))
    dgu = torch.zeros_like(gu)
    dgu[:, :hidden] = dh * u * s * (1 + g * (1 - s))
    dgu[:, up:] = dh * g * s
    dx = (dgu * (1 + e["dgu"])) @ (w1 * (1 + e["w1"]))
    dw1 = (dgu * (1 + e["dgu_t"])).t() @ (x * (1 + e["x_t"]))
    dw2 = (dy * (1 + e["dy_t"])).t() @ (g * s * u * (1 + e["h_t"]))
    return dx, dw1, dw2


@pytest.mark.parametrize("shape", [(70, 200, 300), (256, 384, 512)])
@pytest.mark.parametrize("scale", ["float8_e8m0fnu", "float32"])
def test_slopes(env, shape, scale):
    torch, mlp8 = env
    T, D, H = shape
    layer = mlp8.Mlp8(D, H, scale=getattr(torch, scale), seed=15)
    gen = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(T, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(T, D, generator=gen, device="cuda", dtype=torch.bfloat16) * 1e-3
    layer.forward(x, train=True)
    got = [v.double().cpu() for v in layer.backward(dy)]
    torch.cuda.synchronize()

    up = layer.up
    at = [v.double().cpu() for v in (x, layer.w1, layer.w2)]
    dy = dy.double().cpu()
    wide = (T, up + H)
    e = {k: torch.zeros(*s, dtype=torch.float64, requires_grad=True) for k, s in
         dict(x=(T, D), x_t=(T, D), w1=(up + H, D), w2=(D, H), kept=wide, dgu=wide, dgu_t=wide, h_t=(T, H), dy=(T, D),
              dy_t=(T, D)).items()}
    grads = gradients(torch, *at, dy, H, up, e)
    for i, name in enumerate(("x", "w1", "w2")):
        true = grads[i].detach()
        rnd = torch.randn(true.shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        if name == "w1":
            rnd[H:up] = 0
        d = true + true.norm() / true.numel() ** 0.5 * rnd
        # the loss's slope along d, as differences give it, is the formula's
        step = 1e-4 * at[i].norm() / d.norm()
        ends = [loss(torch, *[v + sign * step * d if j == i else v for j, v in enumerate(at)], dy, H, up)
                for sign in (1, -1)]
        slope = float((ends[0] - ends[1]) / (2 * step))
        assert abs(slope - float((true * d).sum())) < 1e-5 * float(true.norm() * d.norm())
        # and the layer's, within its roundings
        s = torch.autograd.grad((grads[i] * d).sum(), list(e.values()), retain_graph=True, allow_unused=True)
        s = {k: torch.zeros_like(e[k]) if v is None else v for k, v in zip(e, s)}
        one = lambda v, r: r * r * float((v * v).sum())  # noqa: E731
        var = sum(one(s[k], E4M3) for k in ("w1", "w2", "kept", "h_t"))
        for a, b, r in (("x", "x_t", E4M3), ("dgu", "dgu_t", E5M2), ("dy", "dy_t", E5M2)):
            var += max(one(s[a], r) + one(s[b], r), one(s[a] + s[b], r))
        bound = 6 * var ** 0.5 + 0.003 * float(sum(v.abs().sum() for v in s.values()))
        off = abs(float((got[i] * d).sum()) - slope)
        print(name, "slope", slope, "off", off, "bound", bound, flush=True)
        assert off < bound
        assert bound < 0.1 * float(true.norm() * d.norm())     # (what a bound on the norms would give is 0.2)
