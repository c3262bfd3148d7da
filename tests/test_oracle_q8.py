"""The 8-bit oracle against values worked out by hand, torch's casts and differences."""
import numpy as np
import pytest

from oracle import q8


def test_known_codes():
    t = q8.table(q8.E4M3)
    assert (t[0x38], t[0x7E], t[0x01], t[0x08], t[0xB8]) == (1.0, 448.0, 2.0 ** -9, 2.0 ** -6, -1.0)
    assert np.isnan(t[0x7F]) and np.isnan(t[0xFF]) and len(q8.finite_codes(q8.E4M3)) == 127
    t = q8.table(q8.E5M2)
    assert (t[0x3C], t[0x7B], t[0x01], t[0x7C]) == (1.0, 57344.0, 2.0 ** -16, np.inf)
    assert np.isnan(t[0x7D]) and len(q8.finite_codes(q8.E5M2)) == 124


@pytest.mark.parametrize("fmt,name", [(q8.E4M3, "float8_e4m3fn"), (q8.E5M2, "float8_e5m2")])
def test_codes_and_rounding_are_torchs(fmt, name):
    import torch
    dtype = getattr(torch, name)
    codes = torch.arange(256, dtype=torch.uint8)
    theirs = codes.view(dtype).double().numpy()
    np.testing.assert_array_equal(q8.table(fmt), theirs)
    rng = np.random.default_rng(3)
    v = (rng.standard_normal(20000) * np.exp(3 * rng.standard_normal(20000))).astype(np.float32)
    ties = (q8.finite_codes(fmt)[1:] + q8.finite_codes(fmt)[:-1]) / 2
    v = np.concatenate([v, ties, -ties]).astype(np.float32)
    v = v[np.abs(v) <= q8.MOST[fmt]]
    mine = q8.decode(q8.encode(v, fmt), fmt)
    np.testing.assert_array_equal(mine, torch.from_numpy(v).to(dtype).double().numpy())


def test_scales():
    for fmt in (q8.E4M3, q8.E5M2):
        m = q8.MOST[fmt]
        amax = np.array([m, np.nextafter(m, np.inf), m / 2, m * 0.51, 0.0, 1e-44, 3e38])
        s = q8.scale_of(amax, fmt, q8.POW2)
        assert list(s[:6]) == [1.0, 2.0, 0.5, 1.0, 2.0 ** -126, 2.0 ** -126]
        assert s[6] * m >= 3e38 > s[6] * m / 2
        assert q8.scale_of(np.array([m]), fmt, q8.F32)[0] == 1.0


def test_gradient_is_the_slope():
    rng = np.random.default_rng(5)
    g, u, dh = rng.standard_normal((3, 4000)) * np.array([[3.0], [2.0], [1.0]])
    dg, du = q8.swiglu_grad(g, u, dh)
    e = 1e-6
    num_g = dh * (q8.swiglu(g + e, u) - q8.swiglu(g - e, u)) / (2 * e)
    num_u = dh * (q8.swiglu(g, u + e) - q8.swiglu(g, u - e)) / (2 * e)
    # a central difference is off by e^2 / 6 third derivatives and rounding / e
    np.testing.assert_allclose(dg, num_g, rtol=0, atol=1e-8)
    np.testing.assert_allclose(du, num_u, rtol=0, atol=1e-8)
