"""Attention over values whose byte times scale is past fp32's range (rows written near the largest number round up to
such): they reach no row that does not see them.  Tolerances as for other attention over the cache."""
import numpy as np
import pytest

from oracle import attn8, q8
from test_gpu_attn8 import Problem, env  # noqa: F401
from test_gpu_attn8_scores import FORMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("form", FORMS)
def test_hidden_values_past_the_largest_number(env, form, kind, fmt):  # noqa: F811
    """2^128 and 1.75 * 2^128 before the windows and behind the newest token of rows of every form."""
    torch, L = env
    new, group, dim, name = form
    lens = [new + 70, new + 41]
    window = 24
    p = Problem(torch, L, np.random.default_rng(6), [new, new], lens, group=group, dim=dim, name=name, kind=kind, fmt=fmt)
    # the last key but one of the first sequence, and one before the second's last window
    marks = [(0, lens[0] - 2), (1, lens[1] - window - 1)]
    top = np.array([2.0 ** 128, -1.75 * 2.0 ** 128])
    for b, j in marks:
        page, off = attn8.place(p.table[b], j, 16, p.pages)
        p.scales[1][page, :, off] = 1.75 * 2.0 ** 128 / q8.MOST[fmt]
        p.codes[1][page, :, off, :2] = q8.encode(top / p.scales[1][page, 0, off], fmt)
    p.put()
    out, lse = p.run(window=window)
    rows = set()
    for b, j in marks:
        for i in range(new):
            pos = lens[b] - new + i
            if not pos - window < j <= pos:
                rows |= {(b * new + i, h) for h in range(2 * group)}
    p.check(out, lse, window=window, rows=rows)


@pytest.mark.parametrize("form", FORMS)
def test_rows_written_near_the_largest_number(env, form):  # noqa: F811
    """ds_cache8_write makes such a row of 2^128 (1 - 2^-8), which bf16 and fp32 hold; the tokens before it see the rest."""
    torch, L = env
    new, group, dim, name = form
    if new == 1:
        pytest.skip("a prompt of one token hides nothing")
    p = Problem(torch, L, np.random.default_rng(7), [new], [new], group=group, dim=dim, name=name, behind=0)
    k = torch.from_numpy(np.random.default_rng(8).standard_normal((new, 2, dim)).astype(np.float32)).cuda()
    v = k.flip(0).contiguous()
    v[new - 1] = 2.0 ** 128 * (1 - 2.0 ** -8)
    L.ds_cache8_write(p.cache, p.chunk, k, v)
    torch.cuda.synchronize()
    for which, (rows, s) in enumerate(((p.cache.k, p.cache.k_scale), (p.cache.v, p.cache.v_scale))):
        p.codes[which], p.scales[which] = rows.view(torch.uint8).cpu().numpy(), s.double().cpu().numpy()
    assert p.values(1, 0, new)[0][new - 1].max() == 2.0 ** 128
    out, lse = p.run()
    p.check(out, lse, rows={(t, h) for t in range(new - 1) for h in range(2 * group)})
