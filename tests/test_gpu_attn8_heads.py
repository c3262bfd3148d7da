"""Attention of few rows over caches of 4 heads and more, whose workgroups take fours of a sequence's heads on one die as
far as the grid divides, and come in plain order behind that.  Tolerances as for other attention over the cache."""
import numpy as np
import pytest

from oracle import q8
from test_gpu_attn8 import Problem, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [4, 5, 8, 12])
@pytest.mark.parametrize("seqs", [1, 7, 8, 9, 19])
def test_every_head_of_every_sequence(env, heads, seqs):  # noqa: F811
    """One token of each sequence, and few: grids with and without a rest."""
    torch, L = env
    rng = np.random.default_rng(heads + seqs)
    for new, group, name, kind in (([1] * seqs, 2, "bfloat16", q8.POW2), (list(rng.integers(0, 4, seqs - 1)) + [3], 3, "float16", q8.F32)):
        lengths = [int(n) + int(rng.integers(0, 90)) for n in new]
        p = Problem(torch, L, rng, [int(n) for n in new], lengths, heads=heads, group=group, dim=64, name=name, kind=kind)
        p.check(*p.run())


@pytest.mark.parametrize("heads", [4, 8])
def test_split_keys(env, heads):  # noqa: F811
    torch, L = env
    for seqs in (1, 3):
        p = Problem(torch, L, np.random.default_rng(heads), [1] * seqs, [4000, 900, 2100][:seqs], heads=heads, group=2, dim=128, page=64)
        assert L.ds_attn8_work(p.q, p.cache, p.chunk) > 0
        p.check(*p.run())
