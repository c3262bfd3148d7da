"""Rotary positions and rows to and from the paged cache against the 64-bit oracle.

Tolerances.  A turned value is a sum of two products with a cosine and a sine.  Their angle's fraction of a
revolution is off by 2^-26 from its rounding to fp32 and 2^-51 of the whole, times 2 pi; the functions by
2^-22, the products and the sum by three roundings of 2^-24: 2^-20 of |x_a| + |x_b| is above
their sum while the whole is below 2^25 revolutions.  Then half a step of the type.  Rows in 8 bits are
ds_q8_quantize's blocks: codes and powers of two are exact; with an fp32 scale the quotient carries two fp32
roundings, so a code is within half a step and 2^-22 of it.  Rows read back are a product in fp32, rounded twice.
"""
import numpy as np
import pytest

from oracle import attn8, q8

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -133}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a device"
    from paper_2406_20037_amd import _lib
    return torch, _lib


def dtypes(torch):
    return ({q8.E4M3: torch.float8_e4m3fn, q8.E5M2: torch.float8_e5m2},
            {q8.POW2: torch.float8_e8m0fnu, q8.F32: torch.float32})


def typed(torch, x, name):
    t = torch.from_numpy(np.asarray(x, np.float32)).to(getattr(torch, name))
    return t.cuda(), t.double().numpy()


def freqs_of(n, base=10000.0):
    return (base ** (-np.arange(n) / max(1, n))).astype(np.float32)


def check_turned(y, x, pos, freqs, name, pairs=False, scale=1.0, inverse=False):
    want = attn8.rotary(x, pos, freqs, pairs, scale, inverse)
    room = np.abs(attn8.rotary(np.abs(x), np.zeros(len(pos)), freqs, pairs, scale))   # |x_a| and |x_b| times scale
    n = len(freqs)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs else (slice(0, n), slice(n, 2 * n))
    both = room[..., a] + room[..., b]
    lim = np.abs(want) * HALF[name] + TINY[name]
    lim[..., a] += both * 2.0 ** -20
    lim[..., b] += both * 2.0 ** -20
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= lim).all(), float(np.max(err / lim))
    assert np.array_equal(y.double().cpu().numpy()[..., 2 * n:], np.asarray(x)[..., 2 * n:])


SHAPES = [(1, 1, 2, 2), (1, 40, 128, 128), (3, 5, 80, 80), (17, 3, 96, 64), (70, 2, 64, 30), (5, 7, 33, 26),
          (600, 4, 128, 128), (2500, 1, 64, 64), (2, 3, 16, 0), (9, 2, 4096, 4096), (4, 1, 5, 4)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
def test_rotary(env, shape, name):
    torch, L = env
    tokens, heads, dim, turn = shape
    rng = np.random.default_rng(tokens + heads + dim + turn)
    x, exact = typed(torch, rng.standard_normal((tokens, heads, dim)), name)
    pos = rng.integers(-50, 200000, tokens)
    freqs = freqs_of(turn // 2)
    p, f = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freqs).cuda()
    for pairs, inverse, scale in ((0, 0, 1.0), (1, 0, 0.7), (0, 1, 1.3), (1, 1, 1.0)):
        y = torch.full_like(x, float("nan"))
        L.ds_rotary(x, p, f, y, pairs=pairs, scale=scale, inverse=inverse)
        torch.cuda.synchronize()
        check_turned(y, exact, pos, freqs, name, pairs, scale, inverse)
        z = x.clone()
        L.ds_rotary(z, p, f, pairs=pairs, scale=scale, inverse=inverse)                  # in place
        torch.cuda.synchronize()
        assert torch.equal(z, y)


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_rotary_strides(env, name):
    """Queries and keys inside one projection's rows, heads before tokens, unaligned rows, one row for all heads."""
    torch, L = env
    rng = np.random.default_rng(3)
    base, exact = typed(torch, rng.standard_normal((23, 9, 72)), name)
    pos = rng.integers(0, 5000, 23)
    freqs = freqs_of(16)
    p, f = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freqs).cuda()
    for at in ((slice(None), slice(2, 7), slice(0, 64)), (slice(None), slice(0, 9, 2), slice(3, 45)),
               (slice(None), slice(1, 2), slice(8, 72))):
        x = base[at]
        whole = torch.full_like(base, 5.0)
        L.ds_rotary(x, p, f, whole[at])
        torch.cuda.synchronize()
        check_turned(whole[at], exact[at], pos, freqs, name)
        mark = torch.ones_like(base, dtype=torch.bool)
        mark[at] = False
        assert (whole[mark] == 5.0).all()
        turned = torch.empty(x.shape[1], 23, x.shape[2], dtype=x.dtype, device="cuda").transpose(0, 1)
        L.ds_rotary(x, p, f, turned)
        torch.cuda.synchronize()
        assert torch.equal(turned, whole[at])
        one = base.clone()
        L.ds_rotary(one[at], p, f)
        torch.cuda.synchronize()
        assert torch.equal(one[at], whole[at]) and torch.equal(one[mark], base[mark])
    wide = base[:, :1].expand(23, 6, 72)
    y = torch.empty(23, 6, 72, dtype=base.dtype, device="cuda")
    L.ds_rotary(wide, p, f, y)
    torch.cuda.synchronize()
    check_turned(y, np.broadcast_to(exact[:, :1], (23, 6, 72)), pos, freqs, name)


def test_rotary_far(env):
    """Positions to the ends of 32 bits: the angle's fraction is the oracle's, which forms it in 64 bits too."""
    torch, L = env
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 123456789, 2 ** 30 + 7, 0])
    freqs = np.array([2.0 ** -8, 0.75 * 2.0 ** -7, 1e-4, 3.3e-3], np.float32)      # below 2^23 revolutions
    rng = np.random.default_rng(5)
    x, exact = typed(torch, rng.standard_normal((6, 3, 8)), "float32")
    y = torch.empty_like(x)
    L.ds_rotary(x, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freqs).cuda(), y)
    torch.cuda.synchronize()
    check_turned(y, exact, pos, freqs, "float32")


def test_rotary_gradient(env):
    """The inverse is the gradient: against the formula's transpose and against central differences."""
    torch, L = env
    rng = np.random.default_rng(7)
    pos = rng.integers(0, 9000, 11)
    freqs = freqs_of(12)
    p, f = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freqs).cuda()
    for pairs in (False, True):
        x, ex = typed(torch, rng.standard_normal((11, 2, 32)), "float32")
        dy, edy = typed(torch, rng.standard_normal((11, 2, 32)), "float32")
        dx = torch.empty_like(dy)
        L.ds_rotary(dy, p, f, dx, pairs=pairs, scale=1.25, inverse=True)
        torch.cuda.synchronize()
        check_turned(dx, edy, pos, freqs, "float32", pairs, 1.25, True)
        # sum(dy * y(x)) moves along e by sum(dx * e): y is linear, so the difference has no error of its own but
        # y's, 2^-20 of |x_a| + |x_b| each, twice over a step of 2: 2^-20 sum |dy| (|x| + 1)
        for _ in range(4):
            e = rng.standard_normal(x.shape).astype(np.float32)
            up, down = torch.empty_like(x), torch.empty_like(x)
            te = torch.from_numpy(e).cuda()
            L.ds_rotary(x + te, p, f, up, pairs=pairs, scale=1.25)
            L.ds_rotary(x - te, p, f, down, pairs=pairs, scale=1.25)
            torch.cuda.synchronize()
            moved = float((dy.double() * (up.double() - down.double())).sum()) / 2
            want = float((dx.double().cpu().numpy() * e).sum())
            lim = 2.0 ** -18 * 1.25 * float((np.abs(edy).max() * (np.abs(ex) + np.abs(e))).sum())
            assert abs(moved - want) <= lim


# ---- rows ---------------------------------------------------------------------------------

SENTINEL = 0x5B


class Pool:
    """A cache whose every byte is a sentinel, in pages that lie apart, and lists of sequences."""

    def __init__(self, torch, L, rng, new, lengths, *, heads=2, dim=64, page=16, fmt=q8.E4M3, kind=q8.POW2, first=0,
                 extra=3, bad=()):
        f, k = dtypes(torch)
        self.torch, self.L, self.fmt, self.kind = torch, L, fmt, kind
        seqs = len(new)
        cols = max(1, max((-(-n // page) for n in lengths), default=1))
        pages = int(sum(-(-n // page) for n in lengths)) + extra
        order = rng.permutation(pages)
        table = rng.integers(0, pages, (seqs, cols)).astype(np.int32) if seqs else np.zeros((0, 1), np.int32)
        at = 0
        for b, n in enumerate(lengths):
            m = -(-n // page)
            table[b, :m] = order[at:at + m]
            at += m
        for b, col, number in bad:
            table[b, col] = number
        self.starts = (first + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
        self.lengths, self.table = np.asarray(lengths, np.int32), table
        self.tokens = int(self.starts[-1]) + 2
        self.pages, self.page, self.heads, self.dim = pages, page, heads, dim
        gap = 48
        self.store = torch.full((2, pages + 1, heads * page * dim + gap), SENTINEL, dtype=torch.uint8, device="cuda")
        rows = [self.store[i, :pages, :heads * page * dim].view(f[fmt]).unflatten(1, (heads, page, dim)) for i in (0, 1)]
        if kind == q8.POW2:
            self.scales = torch.full((2, pages + 1, heads * page + 5), 200, dtype=torch.uint8, device="cuda")
        else:
            self.scales = torch.full((2, pages + 1, heads * page + 5), 1e30, device="cuda")
        sc = [self.scales[i].view(k[kind])[:pages, :heads * page].unflatten(1, (heads, page)) for i in (0, 1)]
        self.cache = L.Cache8.of(rows[0], rows[1], sc[0], sc[1])
        self.chunk = L.Chunk(*(torch.from_numpy(a).cuda() for a in (self.starts, self.lengths, self.table)))
        self.places = attn8.places(self.starts, self.lengths, self.table, page, pages, self.tokens)

    def codes(self, which):
        """(codes [pages, heads, page, dim], scales) after a look at what lies between."""
        n = self.heads * self.page
        store, sc = self.store[which].cpu().numpy(), self.scales[which].cpu()
        assert (store[self.pages:] == SENTINEL).all() and (store[:, n * self.dim:] == SENTINEL).all()
        filler = sc.flatten()[-1]
        assert (sc[self.pages:] == filler).all() and (sc[:, n:] == filler).all()
        s = sc.numpy().astype(np.float64)
        if self.kind == q8.POW2:
            s = np.ldexp(1.0, sc.numpy().astype(int) - 127)
        shape = (self.pages, self.heads, self.page)
        return store[:self.pages, :n * self.dim].reshape(*shape, self.dim), s[:self.pages, :n].reshape(shape)


def check_rows(pool, which, exact):
    codes, scales = pool.codes(which)
    untouched = np.ones(codes.shape[:3], bool)
    for t, at in enumerate(pool.places):
        if at is None or at[2] is None:
            continue
        page, off = at[2:]
        untouched[page, :, off] = False
        x = exact[t]
        want = attn8.row_scale(x, pool.fmt, pool.kind)
        s = scales[page, :, off]
        if pool.kind == q8.POW2:
            np.testing.assert_array_equal(s, want)
        else:
            assert (np.abs(s - want) <= 2.0 ** -23 * want).all()
        got, by = q8.decode(codes[page, :, off], pool.fmt), s[:, None]
        fin = np.isfinite(x)
        if pool.kind == q8.POW2:
            np.testing.assert_array_equal(got[fin], q8.decode(q8.encode(x / by, pool.fmt), pool.fmt)[fin])
        else:
            v = np.abs(np.where(fin, x, 0.0)) / by
            lim = q8.step_at(np.minimum(v * (1 + 2.0 ** -22), q8.MOST[pool.fmt]), pool.fmt) / 2 + v * 2.0 ** -22
            assert (np.abs(got - x / by) <= lim)[fin].all()
        assert np.isnan(got[np.isnan(x)]).all()
        inf = np.isinf(x)
        assert (np.isnan(got[inf]) if pool.fmt == q8.E4M3 else got[inf] == x[inf]).all()
    filler = SENTINEL
    assert (codes[untouched] == filler).all()
    blank = scales[untouched]
    assert blank.size == 0 or (blank == blank.flat[0]).all() and blank.flat[0] in (2.0 ** 73, np.float32(1e30))


# (new tokens of each sequence, its length, first token of the call)
LISTS = [([1], [1], 0), ([1, 1, 1], [5, 33, 16], 0), ([0, 7, 0, 40, 1], [9, 7, 0, 55, 100], 2),
         ([3, 2], [1, 2], 1), ([130], [130], 0), ([0, 0], [4, 0], 3), ([600, 1, 45], [600, 300, 45], 0)]


@pytest.mark.parametrize("lists", LISTS, ids=str)
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
def test_write_and_read(env, lists, kind, fmt):
    torch, L = env
    new, lengths, first = lists
    for i, (heads, dim, page, name) in enumerate(((1, 128, 16, "bfloat16"), (3, 80, 48, "float32"), (2, 16, 64, "float16"),
                                                  (2, 256, 16, "float32"), (5, 144, 32, "bfloat16"))):
        rng = np.random.default_rng(31 * i + len(new) + 2 * kind + fmt)
        p = Pool(torch, L, rng, new, lengths, heads=heads, dim=dim, page=page, fmt=fmt, kind=kind, first=first)
        vals = [rng.standard_normal((p.tokens, heads, dim)) * np.exp(2 * rng.standard_normal((p.tokens, heads, 1)))
                for _ in range(2)]
        for v in vals:
            v[rng.random(v.shape) < 0.05] = 0.0
            v[p.tokens // 2] = 0.0
        (k, ek), (v, ev) = (typed(torch, x, name) for x in vals)
        L.ds_cache8_write(p.cache, p.chunk, k, v)
        torch.cuda.synchronize()
        check_rows(p, 0, ek)
        check_rows(p, 1, ev)
        back = [torch.full_like(k, 7.0) for _ in range(2)]
        L.ds_cache8_read(p.cache, p.chunk, *back)
        torch.cuda.synchronize()
        for which, out in enumerate(back):
            codes, scales = p.codes(which)
            got = out.double().cpu().numpy()
            for t, at in enumerate(p.places):
                if at is None:
                    assert (got[t] == 7.0).all()
                elif at[2] is None:
                    assert (got[t] == 0.0).all()
                else:
                    want = q8.decode(codes[at[2], :, at[3]], fmt) * scales[at[2], :, at[3]][:, None]
                    lim = np.abs(want) * (HALF[name] + 2.0 ** -24) + TINY[name]
                    assert (np.abs(got[t] - want) <= lim).all()


def test_write_special_values(env):
    torch, L = env
    for fmt in (q8.E4M3, q8.E5M2):
        for kind in (q8.POW2, q8.F32):
            rng = np.random.default_rng(2)
            p = Pool(torch, L, rng, [9], [9], heads=2, dim=32, fmt=fmt, kind=kind)
            x = rng.standard_normal((p.tokens, 2, 32))
            x[0, 0, 3], x[1, 1, 0], x[2, :, 5], x[3] = np.nan, np.inf, -np.inf, np.nan
            x[4] = 1e-42
            x[5, 0, :4] = q8.MOST[fmt], -q8.MOST[fmt], 1e38, 0.0
            x[6, 1] = 2.0 ** -130
            k, ek = typed(torch, x, "float32")
            L.ds_cache8_write(p.cache, p.chunk, k, k)
            torch.cuda.synchronize()
            check_rows(p, 0, ek)
            check_rows(p, 1, ek)


def test_rows_as_quantize_writes_them(env):
    """The same codes and scales as ds_q8_quantize of the rows."""
    torch, L = env
    rng = np.random.default_rng(4)
    for kind in (q8.POW2, q8.F32):
        f, s = dtypes(torch)
        p = Pool(torch, L, rng, [37], [50], heads=1, dim=128, kind=kind)
        k, _ = typed(torch, rng.standard_normal((p.tokens, 1, 128)), "bfloat16")
        L.ds_cache8_write(p.cache, p.chunk, k, k)
        m = L.Q8(p.tokens, 128, scale=s[kind])
        L.ds_q8_quantize(k[:, 0], m)
        torch.cuda.synchronize()
        codes, scales = p.codes(0)
        data, by = m.data.view(torch.uint8).cpu().numpy(), m.scale.float().cpu().numpy()
        for t, at in enumerate(p.places):
            if at is not None:
                assert np.array_equal(codes[at[2], 0, at[3]], data[t]) and scales[at[2], 0, at[3]] == by[t, 0]


def test_bad_pages(env):
    """Numbers outside the cache: nothing is written for them, zeros are read."""
    torch, L = env
    rng = np.random.default_rng(6)
    bad = [(0, 1, -1), (1, 0, 10 ** 6), (1, 2, 2 ** 31 - 1), (2, 0, -2 ** 31)]
    p = Pool(torch, L, rng, [40, 50, 3], [40, 50, 3], bad=bad)
    k, ek = typed(torch, rng.standard_normal((p.tokens, 2, 64)), "bfloat16")
    L.ds_cache8_write(p.cache, p.chunk, k, k)
    out = [torch.full_like(k, 7.0) for _ in range(2)]
    L.ds_cache8_read(p.cache, p.chunk, *out)
    torch.cuda.synchronize()
    check_rows(p, 0, ek)
    got = out[0].float().cpu().numpy()
    for t, at in enumerate(p.places):
        if at is None or at[2] is None:
            assert (got[t] == (7.0 if at is None else 0.0)).all()
        else:
            assert (got[t] != 0.0).any()


def test_many_sequences(env):
    """More sequences than a workgroup keeps in LDS, most of them without a new token."""
    torch, L = env
    rng = np.random.default_rng(8)
    new = rng.integers(0, 2, 2500)
    p = Pool(torch, L, rng, list(new), list(new + rng.integers(0, 3, 2500)), heads=1, dim=16)
    k, ek = typed(torch, rng.standard_normal((p.tokens, 1, 16)), "float32")
    L.ds_cache8_write(p.cache, p.chunk, k, k)
    torch.cuda.synchronize()
    check_rows(p, 0, ek)


def test_rows_strides(env):
    """Keys and values inside one projection's rows, and outputs in heads' order."""
    torch, L = env
    rng = np.random.default_rng(9)
    p = Pool(torch, L, rng, [30, 5], [30, 44], heads=3, dim=48)
    base, exact = typed(torch, rng.standard_normal((p.tokens, 12, 52)), "bfloat16")
    for d in (0, 3):
        k, v = base[:, 1:10:4, d:d + 48], base[:, 9:, d:d + 48]
        L.ds_cache8_write(p.cache, p.chunk, k, v)
        torch.cuda.synchronize()
        check_rows(p, 0, exact[:, 1:10:4, d:d + 48])
        check_rows(p, 1, exact[:, 9:, d:d + 48])
    a = [torch.zeros(p.tokens, 3, 48, device="cuda") for _ in range(2)]
    b = [torch.zeros(3, p.tokens, 48, device="cuda").transpose(0, 1) for _ in range(2)]
    L.ds_cache8_read(p.cache, p.chunk, *a)
    L.ds_cache8_read(p.cache, p.chunk, *b)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_far_pages(env):
    """A cache of more than 2^32 bytes a side: the last page is the one that is written."""
    torch, L = env
    pages, page, dim = 33000, 512, 256
    k8, v8 = (torch.zeros(pages, 1, page, dim, dtype=torch.uint8, device="cuda") for _ in range(2))
    s = [torch.full((pages, 1, page), 1.0, device="cuda") for _ in range(2)]
    cache = L.Cache8.of(*(x.view(torch.float8_e4m3fn) for x in (k8, v8)), *s)
    lists = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 3], [515], [[0, pages - 1]])]
    rng = np.random.default_rng(10)
    k, ek = typed(torch, rng.standard_normal((3, 1, dim)), "float32")
    L.ds_cache8_write(cache, L.Chunk(*lists), k, k)
    back = [torch.empty_like(k) for _ in range(2)]
    L.ds_cache8_read(cache, L.Chunk(*lists), *back)
    torch.cuda.synchronize()
    lim = np.abs(ek).max(-1, keepdims=True) / 448 * 16 + np.abs(ek) * 2.0 ** -22
    assert all((np.abs(b.double().cpu().numpy() - ek) <= lim).all() for b in back)
    assert int((k8[-1, 0, :3] != 0).any(-1).sum()) == 3 and not bool(k8[:-1].any()) and not bool(k8[-1, 0, 3:].any())
