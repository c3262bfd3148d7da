"""Lists that name more tokens than a call has (a batch that is answered in parts): the tokens that are there stand at the
positions that the lists give them, in attention as in the cache.  Tolerances as for other attention over it."""
import numpy as np
import pytest

from test_gpu_attn8 import Problem, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [(5, 3, 2, 64, "bfloat16"), (30, 19, 2, 128, "float16"), (150, 97, 2, 64, "bfloat16"),
                                  (60, 41, 3, 48, "float32"), (90, 55, 2, 192, "bfloat16")], ids=str)
def test_part_of_a_sequence(env, case):  # noqa: F811
    torch, L = env
    new, there, group, dim, name = case
    p = Problem(torch, L, np.random.default_rng(new), [new], [new + 80], group=group, dim=dim, name=name, behind=0)
    for window in (0, 20):
        out, lse = torch.full_like(p.q, 5.0), torch.full(p.q.shape[:2], 5.0, device="cuda")
        L.ds_attn8(p.q[:there], p.cache, p.chunk, out[:there], lse[:there], window=window)
        torch.cuda.synchronize()
        p.check(out, lse, window=window, rows={(t, h) for t in range(there) for h in range(2 * group)})
        assert bool((out[there:] == 5.0).all()) and bool((lse[there:] == 5.0).all())
