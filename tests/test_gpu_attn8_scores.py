"""Attention over the 8-bit cache where its softmax is steep, or has one key: in each of its forms (up to 16 rows a
cache head, up to 32, many; heads wider than 128; fp32 queries).  Tolerances as for other attention over it."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_attn8 import Problem, env  # noqa: F401

pytestmark = pytest.mark.gpu

# (new tokens, query heads a cache head, dim, type)
FORMS = [(1, 4, 64, "bfloat16"), (4, 4, 128, "float16"), (1, 3, 48, "float32"), (2, 5, 192, "bfloat16"),
         (4, 7, 64, "bfloat16"), (9, 3, 128, "float16"), (5, 5, 80, "float32"), (4, 8, 256, "bfloat16"),
         (40, 4, 64, "bfloat16"), (60, 2, 128, "float16"), (70, 2, 96, "bfloat16"), (40, 2, 64, "float32"),
         (33, 3, 160, "bfloat16"), (37, 2, 256, "float16")]


def steep(env, form, kind, factor):  # noqa: F811
    """A sequence whose keys' scales change by `factor` of their place (0 to 1), beside a level one."""
    torch, L = env
    new, group, dim, name = form
    rng = np.random.default_rng(dim + new)
    lens = [max(new, 517), new + 30]
    p = Problem(torch, L, rng, [new, new], lens, group=group, dim=dim, name=name, kind=kind, page=16)
    for j in range(lens[0]):
        s = p.scales[0][p.table[0, j // 16], :, j % 16]
        s *= 2.0 ** round(np.log2(factor(j / lens[0]))) if kind == q8.POW2 else np.float32(factor(j / lens[0]))
        if kind == q8.F32:
            s[:] = s.astype(np.float32)
    p.put()
    return p


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("form", FORMS)
def test_steep_scores(env, form, kind):  # noqa: F811
    """Scores that rise to some hundreds over the keys, fall from there, or jump at one key: the running maximum is
    passed by more than it may lag behind, weights before it vanish, and those after it do."""
    for factor in (lambda x: 1 + 600 * x, lambda x: 1 + 600 * (1 - x), lambda x: 700.0 if 0.7 < x < 0.71 else 1.0):
        p = steep(env, form, kind, factor)
        p.check(*p.run())
        p.check(*p.run(causal=False), causal=False)


@pytest.mark.parametrize("form", FORMS)
def test_scores_of_one_size(env, form):  # noqa: F811
    """Queries of 0 (all weights alike) and a scale of 0, and one of the other sign."""
    torch, L = env
    new, group, dim, name = form
    p = Problem(torch, L, np.random.default_rng(3), [new, 1], [max(new, 100), 40], group=group, dim=dim, name=name)
    p.check(*p.run(scale=0.0), scale=0.0)
    p.check(*p.run(scale=-0.5), scale=-0.5)
    q = p.eq
    p.q.zero_()
    p.eq = 0 * q
    p.check(*p.run())


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
@pytest.mark.parametrize("form", FORMS[:8])
def test_one_key(env, form, fmt):  # noqa: F811
    """A token that sees itself alone is given its value: a scale that is a power of two changes no bit of it."""
    torch, L = env
    _, group, dim, name = form
    for kind in (q8.POW2, q8.F32):
        p = Problem(torch, L, np.random.default_rng(4), [1, 1, 1], [1, 1, 1], group=group, dim=dim, name=name, fmt=fmt, kind=kind)
        out, lse = p.run()
        p.check(out, lse)
        if kind == q8.POW2:
            for b in range(3):
                v, _ = p.values(1, b, 1)
                assert (out[b].double().cpu().numpy() == np.repeat(v[0], group, 0)).all()


@pytest.mark.parametrize("dim", list(range(16, 257, 16)))
def test_every_width(env, dim):  # noqa: F811
    torch, L = env
    for name, kind, new, group in (("bfloat16", q8.POW2, 1, 8), ("float16", q8.F32, 3, 5), ("bfloat16", q8.F32, 5, 6),
                                   ("float16", q8.POW2, 5, 5), ("float16", q8.POW2, 33, 2), ("bfloat16", q8.F32, 33, 2)):
        p = Problem(torch, L, np.random.default_rng(dim), [new, 1], [150, 33], group=group, dim=dim, name=name, kind=kind, page=32)
        p.check(*p.run())


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("form", FORMS)
def test_scales_of_masked_places(env, form, kind):  # noqa: F811
    """A scale that is no number, or infinite, of a key or a value reaches the rows that see it and no others."""
    torch, L = env
    new, group, dim, name = form
    lens = [max(new, 90), max(new, 41)]
    window = 24
    for odd in (np.nan, np.inf)[:1 if kind == q8.POW2 else 2]:
        for which in (0, 1):
            p = Problem(torch, L, np.random.default_rng(6), [new, new], lens, group=group, dim=dim, name=name, kind=kind)
            # the last key but one of the first sequence, and one before the second's last window
            marks = [(0, lens[0] - 2), (1, lens[1] - window - 1)]
            for b, j in marks:
                p.scales[which][p.table[b, j // 16], :, j % 16] = odd
            p.put()
            out, lse = p.run(window=window)
            rows, broken = set(), []
            for b, j in marks:
                for i in range(new):
                    pos = lens[b] - new + i
                    if pos - window < j <= pos:
                        broken.append(b * new + i)
                    else:
                        rows |= {(b * new + i, h) for h in range(2 * group)}
            p.check(out, lse, window=window, rows=rows)
            if kind == q8.F32 and (which == 1 or np.isnan(odd)):
                assert not torch.isfinite(out[broken]).any()


def test_one_page_for_all(env):  # noqa: F811
    """The same page at several places of a table and in two sequences: each place is a key of its own."""
    torch, L = env
    for new, group in ((1, 4), (4, 6), (40, 2)):
        p = Problem(torch, L, np.random.default_rng(8), [new, new], [96, 80], group=group)
        p.table[0, 2] = p.table[0, 0]
        p.table[1, :] = p.table[0, 1]
        p.lists[2].copy_(torch.from_numpy(p.table))
        p.check(*p.run())


def test_windows_past_everything(env):  # noqa: F811
    torch, L = env
    for new, group in ((1, 4), (4, 6), (40, 2)):
        p = Problem(torch, L, np.random.default_rng(9), [new, new], [700, 300], group=group)
        want, lse = p.run()
        for window in (2 ** 31 - 1, 2 ** 31, 2 ** 63 - 1):
            got = p.run(window=window, max_len=2 ** 63 - 1)
            p.check(*got)
            assert torch.equal(got[0], want) and torch.equal(got[1], lse)
