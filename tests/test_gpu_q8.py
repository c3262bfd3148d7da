"""The 8-bit operators against the 64-bit oracle.

Tolerances.  A power-of-two scale and the codes under it are exact, so equal.  With an
fp32 scale the quotient carries two fp32 roundings (2^-23 of it), so a code is within
half a step and 2^-22 of the quotient.  The gated unit's values carry about ten fp32
roundings, 2^-20 of the product (of 1 + |g| where the gate's slope cancels).  A product's fp32 sum of K terms is within (K + 8) 2^-24 of
the sum of magnitudes; through the 8-bit matrix instructions each eight products keep
13 bits below their largest, 8 * 2^-13 of the sum of magnitudes; bf16 and fp16 outputs
round by 2^-9 and 2^-12.
"""
import numpy as np
import pytest

from oracle import q8

pytestmark = pytest.mark.gpu

@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a device"
    from paper_2406_20037_amd import _lib
    return torch, _lib


def dtypes(torch):
    return ({q8.E4M3: torch.float8_e4m3fn, q8.E5M2: torch.float8_e5m2},
            {q8.POW2: torch.float8_e8m0fnu, q8.F32: torch.float32})


SENTINEL = 0x5B


def make(torch, L, rows, cols, fmt=q8.E4M3, kind=q8.POW2, block_rows=1):
    """An empty Q8 whose storage, past the rows' ends too, is filled with a sentinel."""
    f, k = dtypes(torch)
    ld = (cols + 15) // 16 * 16 + 16
    store = torch.full((rows + 1, ld), SENTINEL, dtype=torch.uint8, device="cuda")
    nb = -(-cols // 128)
    sc = torch.full((-(-rows // block_rows) + 1, nb + 3), 200, dtype=torch.uint8, device="cuda").view(k[kind]) \
        if kind == q8.POW2 else torch.full((-(-rows // block_rows) + 1, nb + 3), 1e30, device="cuda")
    m = L.Q8.of(store.view(f[fmt])[:rows, :cols], sc[:-1, :nb], block_rows)
    m.store, m.sc = store, sc
    return m


def got(m):
    """(codes, scale values) of a Q8, after checking that nothing past its edges was written."""
    store = m.store.cpu().numpy()
    assert (store[m.rows:] == SENTINEL).all() and (store[:, m.cols:] == SENTINEL).all()
    edge = m.sc.float().cpu().numpy()
    nr, nc = m.scale.shape
    filler = edge[-1, -1]
    assert (edge[nr:] == filler).all() and (edge[:, nc:] == filler).all()
    return store[: m.rows, : m.cols], edge[:nr, :nc].astype(np.float64)


def check_q8(m, x, fmt, kind, block_rows=1, noise=None):
    """m holds x: exactly the oracle's codes, or, where a scale or the values (by up to
    `noise`) carry fp32 rounding, codes and scales within that."""
    codes, s = got(m)
    fin = np.isfinite(x)
    if kind == q8.POW2 and noise is None:
        v, want, by = q8.quantize(x, fmt, kind, block_rows)
        np.testing.assert_array_equal(s, want)
        np.testing.assert_array_equal(q8.decode(codes, fmt)[fin], q8.decode(q8.encode(v, fmt), fmt)[fin])
        return
    noise = np.zeros_like(x) if noise is None else noise
    mag = np.abs(x)
    lo = q8.scale_of(q8.block_amax(np.maximum(mag - noise, 0), block_rows) * (1 - 2.0 ** -23), fmt, kind)
    hi = q8.scale_of(q8.block_amax(mag + noise, block_rows) * (1 + 2.0 ** -23), fmt, kind)
    assert ((lo <= s) & (s <= hi)).all()
    by = q8.spread(s, *x.shape, block_rows)
    v, off = mag / by, noise / by + mag / by * 2.0 ** -22
    lim = q8.step_at(np.minimum(v + off, q8.MOST[fmt]), fmt) / 2 + off
    err = np.abs(q8.decode(codes, fmt) - x / by)
    assert (err <= lim)[fin].all(), float(np.max((err / lim)[fin]))


def values(rng, rows, cols):
    x = rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    if rows > 2:
        x[rows // 2] = 0.0
    return x


def typed(torch, x, name):
    """(device tensor of the type, its exact values)."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(getattr(torch, name))
    return t.cuda(), t.double().numpy()


SHAPES = [(1, 1), (1, 128), (1, 4096), (2, 129), (16, 64), (127, 255), (128, 128), (129, 257), (300, 1000)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
def test_quantize(env, shape, kind, fmt):
    torch, L = env
    rng = np.random.default_rng(sum(shape) + 7 * kind + fmt)
    for name in ("float32", "float16", "bfloat16"):
        x, exact = typed(torch, values(rng, *shape), name)
        for block_rows in (1, 128):
            for want_row, want_col in ((1, 0), (0, 1), (1, 1)):
                row = make(torch, L, *shape, fmt, kind, block_rows) if want_row else None
                col = make(torch, L, *shape[::-1], fmt, kind, block_rows) if want_col else None
                L.ds_q8_quantize(x, row, col)
                torch.cuda.synchronize()
                if row:
                    check_q8(row, exact, fmt, kind, block_rows)
                if col:
                    check_q8(col, exact.T, fmt, kind, block_rows)


def test_quantize_strides_and_alignment(env):
    torch, L = env
    rng = np.random.default_rng(11)
    for name in ("float32", "bfloat16"):
        base, exact = typed(torch, values(rng, 150, 400), name)
        for rows, cols in ((slice(1, 150), slice(3, 260)), (slice(0, 150, 3), slice(8, 392)),
                           (slice(5, 6), slice(1, 400))):
            x, e = base[rows, cols], exact[rows, cols]
            row, col = make(torch, L, *e.shape), make(torch, L, *e.shape[::-1])
            L.ds_q8_quantize(x, row, col)
            torch.cuda.synchronize()
            check_q8(row, e, q8.E4M3, q8.POW2)
            check_q8(col, e.T, q8.E4M3, q8.POW2)
            alone = make(torch, L, *e.shape)
            L.ds_q8_quantize(x, alone)
            torch.cuda.synchronize()
            check_q8(alone, e, q8.E4M3, q8.POW2)


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
def test_quantize_extremes(env, kind, fmt):
    """Ties, the largest and smallest numbers, and what is not a number beside others."""
    torch, L = env
    vals = q8.finite_codes(fmt)
    ties = (vals[1:] + vals[:-1]) / 2
    x = np.zeros((12, 256))
    x[0, : len(ties)] = ties
    x[0, 255] = vals[-1]
    x[0, 127] = vals[-1]
    x[1] = 3e38
    x[2] = 1e-45
    x[3, ::2], x[3, 1::2] = 1e-40, -3e-39
    x[4, 5], x[4, 6], x[4, 7] = 1.0, 448.0, 448.00003
    x[5], x[5, 3], x[5, 200], x[5, 201] = 2.5, np.nan, np.inf, -np.inf
    x[6] = np.nan
    x[7] = -np.inf
    x[8] = -0.0
    x[9, :128] = 57345.0
    t, e = typed(torch, x, "float32")
    for block_rows in (1, 128):
        row, col = make(torch, L, 12, 256, fmt, kind, block_rows), make(torch, L, 256, 12, fmt, kind, block_rows)
        L.ds_q8_quantize(t, row, col)
        torch.cuda.synchronize()
        for m, v in ((row, e), (col, e.T)):
            check_q8(m, v, fmt, kind, block_rows)
            d = q8.decode(got(m)[0], fmt)
            assert np.isnan(d[np.isnan(v)]).all()
            inf = np.isinf(v)
            assert np.isnan(d[inf]).all() if fmt == q8.E4M3 else (d[inf] == v[inf]).all()
            assert np.isfinite(d[np.isfinite(v)]).all()


def operand(torch, L, rng, rows, cols, fmt, kind, block_rows, spread=2.0):
    """A Q8 of random codes and scales between NaN-coded edges, and its exact values."""
    m = make(torch, L, rows, cols, fmt, kind, block_rows)
    m.store.fill_(0x7F)                               # NaN in both formats
    x = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, cols)) / 2)
    codes = q8.encode(np.clip(x * q8.MOST[fmt] / 64, -q8.MOST[fmt], q8.MOST[fmt]), fmt)
    if rows * cols:
        m.store[:rows, :cols] = torch.from_numpy(codes).cuda()
    nr, nc = m.scale.shape
    e = rng.integers(-12, 5, (nr, nc))
    if kind == q8.POW2:
        s = 2.0 ** e
        m.scale.view(torch.uint8).copy_(torch.from_numpy((e + 127).astype(np.uint8)))
        m.sc.view(torch.uint8)[nr:] = 255
        m.sc.view(torch.uint8)[:, nc:] = 255          # NaN past the edges
    else:
        s = (2.0 ** e * rng.uniform(1, 2, (nr, nc))).astype(np.float32)
        m.scale.copy_(torch.from_numpy(s))
        m.sc[nr:] = float("nan")
        m.sc[:, nc:] = float("nan")
        s = s.astype(np.float64)
    return m, q8.decode(codes, fmt) * q8.spread(s, rows, cols, block_rows)


def check_product(c, a, b, name, rows):
    """c against a b^T under the bounds above."""
    want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
    K = a.shape[1]
    lim = (K + 8) * 2.0 ** -24 * mags + 1e-37
    if name != "float32":
        lim = lim + np.abs(want) * (2.0 ** -8 if name == "bfloat16" else 2.0 ** -11) + \
            (1e-7 if name == "float16" else 0)        # fp16's subnormal step
        if rows > 16:
            lim = lim + 2.0 ** -10 * mags
    out = c.double().cpu().numpy()
    if name == "float16":                             # past 65520 an fp16 is infinite
        over = np.isinf(out) & (np.sign(out) == np.sign(want)) & (np.abs(want) + lim >= 65520)
        out = np.where(over, want, out)
    err = np.abs(out - want)
    assert (err <= lim).all(), (float(np.max(err / lim)), np.argwhere(~(err <= lim))[:4])


MKN = [(1, 1, 1), (1, 128, 16), (1, 4096, 100), (3, 127, 17), (16, 129, 33), (17, 64, 5), (64, 777, 130),
       (100, 1000, 64), (129, 128, 257), (33, 2100, 500), (260, 260, 390), (520, 144, 300)]


@pytest.mark.parametrize("mkn", MKN)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
def test_matmul(env, mkn, kind):
    torch, L = env
    M, K, N = mkn
    rng = np.random.default_rng(M + 3 * K + 5 * N + kind)
    for fa, fb, ra, rb, name in ((0, 0, 1, 128, "bfloat16"), (0, 0, 1, 128, "float32"),
                                 (1, 0, 1, 1, "float32"), (1, 0, 1, 128, "bfloat16"),
                                 (0, 1, 128, 1, "float16"), (1, 1, 1, 1, "bfloat16")):
        print("matmul", mkn, kind, fa, fb, ra, rb, name, flush=True)
        a, av = operand(torch, L, rng, M, K, fa, kind, ra)
        b, bv = operand(torch, L, rng, N, K, fb, kind, rb)
        scale = 1.0
        if name == "float16":                          # keep within its range
            scale = 2.0 ** -12 if fb else 1.0
            bv = bv * scale
            if kind == q8.POW2:
                b.scale.view(torch.uint8).sub_(12)
            else:
                b.scale.mul_(scale)
        c = torch.full((M + 1, N + 3), float("nan"), dtype=getattr(torch, name), device="cuda")
        L.ds_q8_matmul(a, b, c[:M, :N])
        torch.cuda.synchronize()
        check_product(c[:M, :N], av, bv, name, M)
        assert torch.isnan(c[M:]).all() and torch.isnan(c[:, N:]).all(), "wrote past C"


# Shapes that go to each of the other launches: tiles of 256 x 256 and of 256 x 128 (whole,
# ragged and with a reduction that no step of 128 ends), a reduction split over workgroups
# in tiles and under few rows, 32 columns a workgroup.
OTHERS = [(4096, 1024, 4096), (3900, 1000, 4001), (4096, 700, 4096), (2048, 1152, 4096), (2001, 1111, 4000),
          (100, 5000, 200), (300, 2600, 129), (7, 9000, 70), (16, 16300, 33), (3, 300, 8200), (16, 1300, 16390),
          (24, 520, 1000)]


@pytest.mark.parametrize("mkn", OTHERS)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
def test_matmul_every_launch(env, mkn, kind):
    torch, L = env
    M, K, N = mkn
    rng = np.random.default_rng(M + K + N + kind)
    for fa, rb, name in ((0, 128, "bfloat16"), (1, 1, "bfloat16"), (1, 1, "float32")):
        if M * N * K > 1 << 32 and (name == "float32" or (fa and kind)):
            continue                                   # the same launch as smaller shapes
        print("matmul", mkn, kind, fa, rb, name, flush=True)
        a, av = operand(torch, L, rng, M, K, fa, kind, 1)
        b, bv = operand(torch, L, rng, N, K, 0, kind, rb)
        c = torch.full((M + 1, (N + 15) // 8 * 8), float("nan"), dtype=getattr(torch, name), device="cuda")
        L.ds_q8_matmul(a, b, c[:M, :N])
        torch.cuda.synchronize()
        check_product(c[:M, :N], av, bv, name, M)
        assert torch.isnan(c[M:]).all() and torch.isnan(c[:, N:]).all(), "wrote past C"


def test_matmul_scales_in_unaligned_words(env):
    """Scales whose rows do not start at words of four, and a split at such a place."""
    torch, L = env
    rng = np.random.default_rng(41)
    for M, K, N in ((40, 1700, 130), (70, 5000, 64), (300, 900, 260)):
        for name in ("bfloat16", "float32"):
            a, av = operand(torch, L, rng, M, K, 0, q8.POW2, 1)
            b, bv = operand(torch, L, rng, N, K, 0, q8.POW2, 1)
            nb = -(-K // 128)
            for m in (a, b):                           # rows nb bytes apart, from an odd address
                raw = torch.empty(1 + m.rows * nb, dtype=torch.uint8, device="cuda")
                view = raw[1:].view(m.rows, nb)
                view.copy_(m.scale.view(torch.uint8))
                m.tight = L.Q8.of(m.data, view.view(torch.float8_e8m0fnu))
            c = torch.empty(M, N, dtype=getattr(torch, name), device="cuda")
            L.ds_q8_matmul(a.tight, b.tight, c)
            torch.cuda.synchronize()
            check_product(c, av, bv, name, M)


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_matmul_sums_nothing(env, name):
    """K = 0: zeros.  M = 0 or N = 0: nothing is launched."""
    torch, L = env
    for M in (1, 40):
        a, b = L.Q8(M, 0), L.Q8(50, 0)
        c = torch.full((M, 50), 7.0, dtype=getattr(torch, name), device="cuda")
        L.ds_q8_matmul(a, b, c)
        torch.cuda.synchronize()
        assert (c == 0).all()
    L.ds_q8_matmul(L.Q8(0, 64), L.Q8(50, 64), torch.empty(0, 50, device="cuda"))
    L.ds_q8_matmul(L.Q8(5, 64), L.Q8(0, 64), torch.empty(5, 0, device="cuda"))


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("M,name", [(5, "bfloat16"), (70, "bfloat16"), (70, "float32"), (300, "bfloat16")])
def test_matmul_nan_stays_in_its_row_and_column(env, kind, M, name):
    torch, L = env
    rng = np.random.default_rng(17)
    a, av = operand(torch, L, rng, M, 200, q8.E4M3, kind, 1)
    b, bv = operand(torch, L, rng, 140, 200, q8.E4M3, kind, 1)
    a.store[3, 77] = 0x7F
    b.store[139, 199] = 0xFF
    c = torch.empty(M, 140, dtype=getattr(torch, name), device="cuda")
    L.ds_q8_matmul(a, b, c)
    torch.cuda.synchronize()
    bad = torch.isnan(c).cpu().numpy()
    assert bad[3].all() and bad[:, 139].all()
    bad[3], bad[:, 139] = False, False
    assert not bad.any()


def test_matmul_scales_far_apart(env):
    """Blocks of one reduction whose scales differ by 2^60 and exponents at the ends of the range."""
    torch, L = env
    rng = np.random.default_rng(23)
    for M in (4, 40):
        for name in ("bfloat16", "float32"):
            a, av = operand(torch, L, rng, M, 512, q8.E4M3, q8.POW2, 1)
            b, bv = operand(torch, L, rng, 48, 512, q8.E4M3, q8.POW2, 128)
            codes_a, codes_b = (q8.decode(m.store[: m.rows, : m.cols].cpu().numpy(), q8.E4M3) for m in (a, b))
            ea = np.tile(np.array([97, 127, 157, 1]), (M, 1))
            eb = np.tile(np.array([127, 120, 127, 250]), (1, 1))
            a.scale.view(torch.uint8).copy_(torch.from_numpy(ea.astype(np.uint8)))
            b.scale.view(torch.uint8).copy_(torch.from_numpy(eb.astype(np.uint8)))
            c = torch.empty(M, 48, dtype=getattr(torch, name), device="cuda")
            L.ds_q8_matmul(a, b, c)
            torch.cuda.synchronize()
            check_product(c, codes_a * q8.spread(2.0 ** (ea - 127.0), M, 512),
                          codes_b * q8.spread(2.0 ** (eb - 127.0), 48, 512, 128), name, M)


def test_matmul_gradients_are_the_slopes(env):
    """With L = sum(C * G): dA = G B and dB = G^T A by the same call on transposes, against the
    change of L along a direction, which is exact for a bilinear form."""
    torch, L = env
    rng = np.random.default_rng(29)
    M, N, K = 70, 90, 150
    f, k = dtypes(torch)

    def both(x, fmt=q8.E4M3):
        t = torch.from_numpy(x.astype(np.float32)).cuda()
        r, c = L.Q8(*x.shape, f[fmt]), L.Q8(*x.shape[::-1], f[fmt])
        L.ds_q8_quantize(t, r, c)
        return r, c

    A, B, G = rng.standard_normal((M, K)), rng.standard_normal((N, K)), rng.standard_normal((M, N))
    a, a_t = both(A)
    b, b_t = both(B)
    g, g_t = both(G, q8.E5M2)
    dA, dB = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    L.ds_q8_matmul(g, b_t, dA)
    L.ds_q8_matmul(g_t, a_t, dB)
    val = {n: m.values().double().cpu().numpy() for n, m in
           dict(a_t=a_t, b_t=b_t, g=g, g_t=g_t).items()}
    for grad, lhs, rhs, x in ((dA, val["g"], val["b_t"].T, A), (dB, val["g_t"], val["a_t"].T, B)):
        D = rng.standard_normal(x.shape)
        slope = np.sum(((x + D) @ rhs.T) * lhs) - np.sum((x @ rhs.T) * lhs)
        gradient = grad.double().cpu().numpy()
        mags = np.abs(lhs) @ np.abs(rhs)
        assert np.abs(np.sum(gradient * D) - slope) <= \
            (lhs.shape[1] + 8) * 2.0 ** -24 * np.sum(mags * np.abs(D)) + 1e-9 * np.sum(mags)


def gated(torch, rng, rows, hidden, up, name):
    gu = rng.standard_normal((rows, up + hidden)) * np.exp(rng.standard_normal((rows, 1)))
    gu[:, hidden:up] = np.nan                          # not read
    if hidden > 8:
        gu[0, :8] = [0.0, -0.0, 30.0, -30.0, 88.0, -88.0, 100.0, -200.0]
    t, e = typed(torch, gu, name)
    return t, e[:, :hidden], e[:, up:]


def unit_noise(g, u):
    """2^-20 of silu(g) u, and what fp32 has no numbers for."""
    return 2.0 ** -20 * np.abs(q8.swiglu(g, u)) + 1e-36 * (1 + np.abs(u))


GATED = [(1, 1, 128), (1, 2048, 2048), (3, 100, 128), (5, 100, 384), (130, 129, 256), (257, 640, 640)]


@pytest.mark.parametrize("shape", GATED)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
def test_swiglu(env, shape, kind, name):
    torch, L = env
    rows, hidden, up = shape
    rng = np.random.default_rng(rows + hidden + kind)
    gu, g, u = gated(torch, rng, rows, hidden, up, name)
    for save in (True, False):
        h = make(torch, L, rows, hidden, q8.E4M3, kind)
        saved = make(torch, L, rows, up + hidden, q8.E4M3, kind) if save else None
        L.ds_swiglu8(gu, h, saved)
        torch.cuda.synchronize()
        check_q8(h, q8.swiglu(g, u), q8.E4M3, kind, noise=unit_noise(g, u))
        if save:
            full = np.zeros((rows, up + hidden))
            full[:, :hidden], full[:, up:] = g, u
            check_q8(saved, full, q8.E4M3, kind)


@pytest.mark.parametrize("shape", GATED)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
def test_swiglu_grad(env, shape, kind, name):
    torch, L = env
    rows, hidden, up = shape
    rng = np.random.default_rng(rows + 2 * hidden + kind)
    saved, v = operand(torch, L, rng, rows, up + hidden, q8.E4M3, q8.POW2 if kind else q8.F32, 1, 1.0)
    # scales that leave gates within +-30 or so
    if saved.scale.dtype == torch.float32:
        saved.scale.mul_(2.0 ** -4)
        v = v * 2.0 ** -4
    else:
        saved.scale.view(torch.uint8).sub_(4)
        v = v * 2.0 ** -4
    dh, d = typed(torch, rng.standard_normal((rows, hidden)) * np.exp(rng.standard_normal((rows, 1))), name)
    g, u = v[:, :hidden], v[:, up:]
    dg, du = q8.swiglu_grad(g, u, d)
    full = np.zeros((rows, up + hidden))
    full[:, :hidden], full[:, up:] = dg, du
    # 1 + g (1 - s) passes 0 near g = -1.28, so its rounding is relative to 1 + |g|
    noise = np.zeros_like(full)
    noise[:, :hidden] = 2.0 ** -20 * np.abs(d * u) * q8.sigmoid(g) * (1 + np.abs(g))
    noise[:, up:] = 2.0 ** -20 * np.abs(du)
    noise += 1e-36 * (1 + np.max(np.abs(d), initial=0) * (1 + np.max(np.abs(u), initial=0)))
    for fmt in (q8.E4M3, q8.E5M2):
        for which in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
            dgu = make(torch, L, rows, up + hidden, fmt, kind) if which[0] else None
            dgu_t = make(torch, L, up + hidden, rows, fmt, kind) if which[1] else None
            h_t = make(torch, L, hidden, rows, q8.E4M3, kind) if which[2] else None
            L.ds_swiglu8_grad(saved, dh, dgu, dgu_t, h_t)
            torch.cuda.synchronize()
            if dgu:
                check_q8(dgu, full, fmt, kind, noise=noise)
            if dgu_t:
                check_q8(dgu_t, full.T, fmt, kind, noise=noise.T)
            if h_t:
                check_q8(h_t, q8.swiglu(g, u).T, q8.E4M3, kind, noise=unit_noise(g, u).T)


def test_empty(env):
    torch, L = env
    for shape in ((0, 5), (5, 0)):
        L.ds_q8_quantize(torch.empty(shape, device="cuda"), L.Q8(*shape), L.Q8(*shape[::-1]))
    L.ds_swiglu8(torch.empty(0, 256, device="cuda"), L.Q8(0, 128))
    saved = make(torch, L, 3, 128)
    L.ds_swiglu8(torch.empty(3, 128, device="cuda"), L.Q8(3, 0), saved)   # nothing but the columns between
    torch.cuda.synchronize()
    assert (got(saved)[0] == 0).all()


def test_two_calls_give_the_same_bits(env):
    torch, L = env
    rng = np.random.default_rng(31)
    for M, K, N, name in ((1, 4000, 70, "bfloat16"), (40, 8192, 64, "float32"),
                          (40, 8192, 64, "bfloat16"), (300, 5000, 200, "bfloat16")):
        a, _ = operand(torch, L, rng, M, K, 0, q8.POW2, 1)
        b, _ = operand(torch, L, rng, N, K, 0, q8.POW2, 128)
        cs = [torch.empty(M, N, dtype=getattr(torch, name), device="cuda") for _ in range(3)]
        for c in cs:
            L.ds_q8_matmul(a, b, c)
        torch.cuda.synchronize()
        assert torch.equal(cs[0], cs[1]) and torch.equal(cs[0], cs[2])


def test_streams_and_graphs(env):
    """A layer's calls on a stream of its own and replayed from a graph, with eager work between."""
    torch, L = env
    rng = np.random.default_rng(37)
    T, D, H = 48, 4096, 200
    up = 256
    x = torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).cuda().bfloat16()
    w, _ = operand(torch, L, rng, up + H, D, 0, q8.POW2, 128, 1.0)
    st = torch.cuda.Stream()

    def layer(s):
        L.ds_q8_quantize(x, x8, x8_t, stream=s)
        L.ds_q8_matmul(x8, w, gu, stream=s)
        L.ds_swiglu8(gu, h, saved, stream=s)
        L.ds_swiglu8_grad(saved, gu[:, :H], dgu, dgu_t, h_t, stream=s)

    x8, x8_t, h = L.Q8(T, D), L.Q8(D, T), L.Q8(T, H)
    saved, dgu, dgu_t, h_t = L.Q8(T, up + H), L.Q8(T, up + H), L.Q8(up + H, T), L.Q8(H, T)
    gu = torch.empty(T, up + H, dtype=torch.bfloat16, device="cuda")
    outs = lambda: [gu.clone()] + [v.view(torch.uint8).clone() for m in (x8, x8_t, h, saved, dgu, dgu_t, h_t)  # noqa: E731
                                   for v in (m.data, m.scale)]
    layer(None)
    torch.cuda.synchronize()
    want = outs()
    st.wait_stream(torch.cuda.current_stream())
    layer(st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, outs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        layer(None)
    for i in range(4):
        for m in (x8, x8_t, h, saved, dgu, dgu_t, h_t):
            m.data.view(torch.uint8).fill_(i)
        gu.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, outs())), i
        layer(None)
        torch.cuda.synchronize()
