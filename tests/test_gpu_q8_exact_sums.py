"""8-bit products of small whole numbers, whose sums every kernel has to give exactly: values in {-1, 0, 1}
and scales of 1 and 2 a block, so that no sum passes 2048, up to where fp16 holds every whole number, and no
group of products needs more bits than the 8-bit instructions keep.  One product left out, or taken twice, shows."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_q8 import env, make  # noqa: F401

pytestmark = pytest.mark.gpu

ONE = {q8.E4M3: 0x38, q8.E5M2: 0x3C}


def whole(torch, L, rng, rows, cols, fmt, kind, block_rows):
    """A Q8 of such values between NaN-coded edges, and the values."""
    m = make(torch, L, rows, cols, fmt, kind, block_rows)
    m.store.fill_(0x7F)
    v = rng.integers(-1, 2, (rows, cols)).astype(np.int8)
    codes = np.where(v == 0, 0, ONE[fmt] | np.where(v < 0, 0x80, 0)).astype(np.uint8)
    m.store[:rows, :cols] = torch.from_numpy(codes).cuda()
    e = rng.integers(0, 2, tuple(m.scale.shape))
    if kind == q8.POW2:
        m.sc.view(torch.uint8)[:] = 255
        m.scale.view(torch.uint8).copy_(torch.from_numpy((127 + e).astype(np.uint8)))
    else:
        m.sc[:] = float("nan")
        m.scale.copy_(torch.from_numpy((2.0 ** e).astype(np.float32)))
    return m, (v * q8.spread(2.0 ** e, rows, cols, block_rows)).astype(np.float32)


# one row to 32, tiles of 128 x 128 (whole, ragged, split), of 256 x 256 and of 256 x 128 (long
# reductions), and reductions that end inside a step, inside 16 bytes, and after less than one step
SHAPES = [(1, 4000, 70), (9, 8200, 300), (31, 1001, 8300), (40, 4100, 130), (128, 128, 128), (130, 77, 260),
          (256, 1111, 384), (1003, 777, 1501), (100, 5000, 200), (2048, 1152, 4096), (2001, 1111, 4000),
          (4096, 1024, 4096), (3900, 1003, 4001), (300, 12901, 11100)]


@pytest.mark.parametrize("mkn", SHAPES)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
def test_sums_are_exact(env, mkn, kind):  # noqa: F811
    torch, L = env
    M, K, N = mkn
    rng = np.random.default_rng(M + 3 * K + N + kind)
    for fa, fb, ra, rb, name in ((0, 0, 1, 128, "float16"), (1, 0, 1, 1, "float32"), (0, 1, 128, 1, "float16")):
        print("exact sums", mkn, kind, fa, fb, ra, rb, name, flush=True)
        a, av = whole(torch, L, rng, M, K, fa, kind, ra)
        b, bv = whole(torch, L, rng, N, K, fb, kind, rb)
        want = av @ bv.T                               # whole numbers below 2^24: exact in fp32
        assert np.max(np.abs(want)) <= 2048
        c = torch.full((M + 1, (N + 15) // 8 * 8), float("nan"), dtype=getattr(torch, name), device="cuda")
        L.ds_q8_matmul(a, b, c[:M, :N])
        torch.cuda.synchronize()
        np.testing.assert_array_equal(c[:M, :N].float().cpu().numpy(), want)
        assert torch.isnan(c[M:]).all() and torch.isnan(c[:, N:]).all(), "wrote past C"


@pytest.mark.parametrize("mkn", [(33, 300, 64), (130, 1003, 260), (70, 5000, 64), (200, 640, 130)])
@pytest.mark.parametrize("tight", [False, True])
def test_scales_past_two_to_the_forty(env, mkn, tight):  # noqa: F811
    """Scales of 2^90 in a few rows of one operand and of 2^-30 in the other; rows of scales that do
    and do not start at words of four."""
    torch, L = env
    M, K, N = mkn
    rng = np.random.default_rng(M + K + N + tight)
    a, av = whole(torch, L, rng, M, K, q8.E4M3, q8.POW2, 1)
    b, bv = whole(torch, L, rng, N, K, q8.E5M2, q8.POW2, 1)
    rows = rng.integers(0, min(M, 128), 3)
    a.scale.view(torch.uint8)[rows] += 90
    av[rows] *= 2.0 ** 90
    a.scale.view(torch.uint8)[rows[0], 0] -= 90
    av[rows[0], :128] *= 2.0 ** -90
    b.scale.view(torch.uint8)[:] -= 30
    want = av.astype(np.float64) @ (bv.astype(np.float64) * 2.0 ** -30).T
    if tight:
        nb = -(-K // 128)
        for m in (a, b):
            raw = torch.empty(1 + m.rows * nb, dtype=torch.uint8, device="cuda")
            view = raw[1:].view(m.rows, nb)
            view.copy_(m.scale.view(torch.uint8))
            m.tight = L.Q8.of(m.data, view.view(torch.float8_e8m0fnu))
        a, b = a.tight, b.tight
    c = torch.empty(M, N, device="cuda")
    L.ds_q8_matmul(a, b, c)
    torch.cuda.synchronize()
    # rows[0] mixes 2^90 and 1: its sums are rounded to fp32 at most once a block
    got, lim = c.double().cpu().numpy(), np.zeros((M, N))
    lim[rows[0]] = (K // 128 + 2) * 2.0 ** -24 * (np.abs(av[rows[0]]).astype(np.float64) @ np.abs(bv).T * 2.0 ** -30)
    assert (np.abs(got - want) <= lim).all()


@pytest.mark.parametrize("mkn", [(5, 1000, 70), (24, 1000, 70), (24, 4300, 64), (40, 1000, 130), (300, 1003, 260), (1030, 640, 2050)])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_sums_that_cancel(env, mkn, kind, block_rows):  # noqa: F811
    """Products of +-256 that sum to 0 beside products of +-2^-6: every partial sum is a multiple of 2^-6 below
    2^18, exact in fp32 in any order, and the sums are exact in 16 bits; 14 bits below the largest product
    would leave nothing of them."""
    torch, L = env
    M, K, N = mkn
    rng = np.random.default_rng(M + K + N + kind + block_rows)
    large = np.arange(K) % 4 < 2                       # pairs of them, and of small ones
    av, bv = rng.integers(-1, 2, (M, K)).astype(np.float64), rng.integers(-1, 2, (N, K)) * 2.0 ** -6
    sign = np.where(rng.random((N, K)) < 0.5, 1.0, -1.0)
    sign[:, 1::2] = -sign[:, 0:K - K % 2:2]
    bv[:, large] = 256.0 * sign[:, large]
    av[:, large] = 1.0
    av[:, K - K % 4:] = 0.0                            # no pair there
    a, b = make(torch, L, M, K, q8.E4M3, kind), make(torch, L, N, K, q8.E4M3, kind, block_rows)
    for m, v in ((a, av), (b, bv)):
        m.store[:m.rows, :m.cols] = torch.from_numpy(q8.encode(v, q8.E4M3)).cuda()
        m.scale.fill_(1.0) if kind == q8.F32 else m.scale.view(torch.uint8).fill_(127)
    want = av @ bv.T
    assert np.max(np.abs(want)) <= 2 and np.any(want)
    few = M <= (32 if K <= 4096 else 16)               # exact without asking
    for name, exact in (("bfloat16", True), ("float16", True), ("bfloat16", False), ("float32", False)):
        if not exact and name == "bfloat16" and not few:
            continue
        c = torch.empty(M, N, dtype=getattr(torch, name), device="cuda")
        L.ds_q8_matmul(a, b, c, exact=exact)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(c.double().cpu().numpy(), want)
