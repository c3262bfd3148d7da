"""Infinities in keys and values (of e5m2) that rows see, in every form of attention over the cache: what the sums of
the definition come to, whatever parts queries and weights are taken in.  Tolerances as for other attention over it."""
import numpy as np
import pytest

from oracle import attn8, q8
from test_gpu_attn8 import Problem, env  # noqa: F401
from test_gpu_attn8_scores import FORMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("form", FORMS)
def test_values(env, form, kind, exact):  # noqa: F811
    """A column with an infinity is infinite, with two of either sign no number; the others are as without."""
    torch, L = env
    new, group, dim, name = form
    length = new + 150
    p = Problem(torch, L, np.random.default_rng(9), [new], [length], group=group, dim=dim, name=name, kind=kind, fmt=q8.E5M2)
    # (of keys that all rows see, weights whose parts are of either sign or 0)
    marks = [(3, 1, 0x7C), (40, 5, 0xFC), (41, 7, 0x7C), (90, 7, 0xFC), (91, 5, 0xFC)]
    want = {1: np.inf, 5: -np.inf, 7: np.nan}
    for j, d, code in marks:
        page, off = attn8.place(p.table[0], j, 16, p.pages)
        p.codes[1][page, :, off, d] = code
    p.put()
    out, lse = p.run(exact=exact)
    got, sums = out.double().cpu().numpy(), lse.double().cpu().numpy()
    (k, _), (v, _) = p.values(0, 0, length), p.values(1, 0, length)
    v = np.where(np.isfinite(v), v, 0.0)
    for i in range(new):
        sees = np.arange(length) <= length - new + i
        for h in range(2 * group):
            row, lim, total, off = p.row(p.eq[i, h], k[:, h // group], v[:, h // group], sees, dim ** -0.5)
            assert abs(sums[i, h] - total) <= off
            for d in range(dim):
                if d in want:
                    np.testing.assert_equal(got[i, h, d], want[d], err_msg=str((i, h, d)))
                else:
                    assert abs(got[i, h, d] - row[d]) <= lim[d], (i, h, d)


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("form", FORMS)
def test_keys(env, form, kind):  # noqa: F811
    """A score of minus infinity has no weight; one of plus infinity leaves a row no number."""
    torch, L = env
    new, group, dim, name = form
    length = new + 150
    p = Problem(torch, L, np.random.default_rng(10), [new], [length], group=group, dim=dim, name=name, kind=kind, fmt=q8.E5M2)
    marks = [5, 60]
    for j in marks:
        page, off = attn8.place(p.table[0], j, 16, p.pages)
        p.codes[0][page, :, off, 2] = 0x7C
    p.put()
    # by the sign of value 2 of a query: bits that take one part, two and three
    p.eq[..., 2] = np.where(np.arange(2 * group) % 2 == 0, -1.0, 1.0) * np.where(np.arange(p.tokens)[:, None] % 2, 1.0, 1.25 + 2.0 ** -20)
    p.q.copy_(torch.from_numpy(p.eq))
    p.eq = p.q.double().cpu().numpy()
    out, lse = p.run()
    got, sums = out.double().cpu().numpy(), lse.double().cpu().numpy()
    (k, _), (v, _) = p.values(0, 0, length), p.values(1, 0, length)
    for i in range(new):
        sees = np.arange(length) <= length - new + i
        sees[marks] = False
        for h in range(2 * group):
            if p.eq[i, h, 2] > 0:
                assert np.isnan(got[i, h]).all() and np.isnan(sums[i, h]), (i, h)
                continue
            row, lim, total, off = p.row(p.eq[i, h], k[:, h // group], v[:, h // group], sees, dim ** -0.5)
            assert abs(sums[i, h] - total) <= off and (np.abs(got[i, h] - row) <= lim).all(), (i, h)
