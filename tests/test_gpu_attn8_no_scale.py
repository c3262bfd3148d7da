"""A power-of-two scale whose byte is 255 is no number: rows read back are none, and so are the rows of attention that see
such a key or value, in every form."""
import numpy as np
import pytest

from oracle import attn8, q8
from test_gpu_attn8 import Problem, env  # noqa: F401
from test_gpu_attn8_scores import FORMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
@pytest.mark.parametrize("name", ["float32", "float16", "bfloat16"])
def test_read(env, name, fmt):  # noqa: F811
    torch, L = env
    p = Problem(torch, L, np.random.default_rng(1), [40], [40], dim=80, name=name, fmt=fmt)
    page, off = attn8.place(p.table[0], 7, 16, p.pages)
    p.scales[0][page, 1, off] = np.nan
    p.codes[0][page, 1, off, :3] = 0
    p.put()
    k, v = (torch.zeros(p.tokens, 2, 80, dtype=p.q.dtype, device="cuda") for _ in range(2))
    L.ds_cache8_read(p.cache, p.chunk, k, v)
    torch.cuda.synchronize()
    none = torch.isnan(k)
    assert none[7, 1].all() and int(none.sum()) == 80 and not torch.isnan(v).any()


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("form", FORMS)
def test_attention(env, form, which):  # noqa: F811
    torch, L = env
    new, group, dim, name = form
    for j in (3, new + 149 - (new > 1)):            # a key that all rows see, and one that the first ones do not
        p = Problem(torch, L, np.random.default_rng(2), [new], [new + 150], group=group, dim=dim, name=name)
        page, off = attn8.place(p.table[0], j, 16, p.pages)
        p.scales[which][page, :, off] = np.nan
        p.codes[which][page, :, off, ::2] = 0       # (and 0 times it)
        p.put()
        out, lse = p.run()
        see = [i for i in range(new) if j <= 150 + i]
        assert torch.isnan(out[see]).all()
        assert torch.isnan(lse[see]).all() if which == 0 else torch.isfinite(lse[see]).all()
        p.check(out, lse, rows={(i, h) for i in range(new) if i not in see for h in range(2 * group)})
