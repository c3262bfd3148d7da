"""Matrices of whole 128 x 128 tiles with 16-byte aligned rows, which have kernels of their own, against
the 64-bit oracle; with the tolerances of the other 8-bit tests, derived there."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_q8 import check_q8, env, make, typed, unit_noise, values  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(128, 256), (384, 128)])
@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_whole(env, shape, name, kind, block_rows):  # noqa: F811
    torch, L = env
    rng = np.random.default_rng(sum(shape) + kind + block_rows)
    for shift in (0, 1):                               # rows from an odd column on, too
        wide, e = typed(torch, values(rng, shape[0], shape[1] + shift), name)
        x, e = wide[:, shift:], e[:, shift:]
        for fmt in (q8.E4M3, q8.E5M2):
            for want_row, want_col in ((0, 1), (1, 1)):
                row = make(torch, L, *shape, fmt, kind, block_rows) if want_row else None
                col = make(torch, L, *shape[::-1], fmt, kind, block_rows) if want_col else None
                L.ds_q8_quantize(x, row, col)
                torch.cuda.synchronize()
                if row:
                    check_q8(row, e, fmt, kind, block_rows)
                if col:
                    check_q8(col, e.T, fmt, kind, block_rows)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_quantize_whole_not_finite(env, bad):  # noqa: F811
    torch, L = env
    rng = np.random.default_rng(5)
    v = values(rng, 256, 256)
    v[3, 200] = v[131, 7] = v[255, 255] = bad
    x, e = typed(torch, v, "bfloat16")
    row, col = make(torch, L, 256, 256), make(torch, L, 256, 256)
    L.ds_q8_quantize(x, row, col)
    torch.cuda.synchronize()
    check_q8(row, e, q8.E4M3, q8.POW2)
    check_q8(col, e.T, q8.E4M3, q8.POW2)


@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("shape", [(128, 128), (256, 384)])
def test_swiglu_grad_whole(env, name, kind, shape):  # noqa: F811
    torch, L = env
    rows, hidden = shape
    rng = np.random.default_rng(rows + hidden + kind)
    saved = make(torch, L, rows, 2 * hidden, q8.E4M3, kind)
    g, e = typed(torch, 4 * rng.standard_normal((rows, 2 * hidden)), name)
    L.ds_q8_quantize(g, saved, None)
    torch.cuda.synchronize()
    v = saved.values().double().cpu().numpy()
    dh, d = typed(torch, rng.standard_normal((rows, hidden)) * np.exp(rng.standard_normal((rows, 1))), name)
    g, u = v[:, :hidden], v[:, hidden:]
    full = np.concatenate(q8.swiglu_grad(g, u, d), 1)
    noise = 2.0 ** -20 * np.abs(full)
    noise[:, :hidden] = 2.0 ** -20 * np.abs(d * u) * q8.sigmoid(g) * (1 + np.abs(g))
    noise += 1e-36 * (1 + np.max(np.abs(d)) * (1 + np.max(np.abs(u))))
    for fmt in (q8.E4M3, q8.E5M2):
        dgu, dgu_t = make(torch, L, rows, 2 * hidden, fmt, kind), make(torch, L, 2 * hidden, rows, fmt, kind)
        h_t = make(torch, L, hidden, rows, q8.E4M3, kind)
        L.ds_swiglu8_grad(saved, dh, dgu, dgu_t, h_t)
        torch.cuda.synchronize()
        check_q8(dgu, full, fmt, kind, noise=noise)
        check_q8(dgu_t, full.T, fmt, kind, noise=noise.T)
        check_q8(h_t, q8.swiglu(g, u).T, q8.E4M3, kind, noise=unit_noise(g, u).T)
