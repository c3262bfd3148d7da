"""How exactly weights enter the product with values, in every form of attention over the cache: by the types alone,
whatever else is in the call.  Tolerances as for other attention over it, with a weight's rounding as it says here."""
import numpy as np
import pytest

import test_gpu_attn8
from oracle import q8
from test_gpu_attn8 import HALF, Problem, env  # noqa: F401
from test_gpu_attn8_scores import FORMS, steep

pytestmark = pytest.mark.gpu

TWO = 2.0 ** -16          # two parts of bf16: the second one's rounding


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
@pytest.mark.parametrize("form", FORMS)
def test_first_tokens(env, form, fmt):  # noqa: F811
    """The first token of a prompt sees itself alone, among rows of every form.  It is given its value: with scales that are
    powers of two to the bit, as no weight is rounded but 1 (in fp32 that of one product, 2^-24, too); else a weight times a
    scale in two parts (three for fp32), an exponential and a quotient off by 2^-20, and the output's half a step."""
    torch, L = env
    new, group, dim, name = form
    for kind in (q8.POW2, q8.F32):
        p = Problem(torch, L, np.random.default_rng(14), [new, new], [new, new], group=group, dim=dim, name=name, fmt=fmt, kind=kind)
        out, _ = p.run()
        for b in range(2):
            v, _ = p.values(1, b, 1)
            v = np.repeat(v[0], group, 0)
            err = np.abs(out[b * new].double().cpu().numpy() - v)
            if kind == q8.POW2:
                lim = np.abs(v) * (2.0 ** -23 if name == "float32" else 0.0)
            else:
                lim = np.abs(v) * (HALF[name] + 2.0 ** -20 + (2.0 ** -24 if name == "float32" else TWO))
            assert (err <= lim).all(), (b, kind, float((err / np.abs(v)).max()))


@pytest.mark.parametrize("form", [f for f in FORMS if f[3] == "bfloat16"])
def test_fp32_scales(env, form, monkeypatch):  # noqa: F811
    """Rows of many keys, of steep scores, and of one key that outweighs the others by less than a running maximum may lag
    behind: two parts for bf16 queries too."""
    monkeypatch.setitem(test_gpu_attn8.WEIGHT, "bfloat16", TWO)
    for factor in (lambda x: 1.0, lambda x: 1 + 600 * x, lambda x: 9.0 if 0.7 < x < 0.71 else 1.0):
        p = steep(env, form, q8.F32, factor)
        p.check(*p.run())


@pytest.mark.parametrize("form", FORMS)
def test_exact(env, form, monkeypatch):  # noqa: F811
    """bf16 queries over powers of two take two parts if the caller asks; where there are as many anyway, nothing changes."""
    torch, L = env
    monkeypatch.setitem(test_gpu_attn8.WEIGHT, "bfloat16", TWO)
    for factor in (lambda x: 1.0, lambda x: 1 + 600 * x, lambda x: 8.0 if 0.7 < x < 0.71 else 1.0):
        p = steep(env, form, q8.POW2, factor)
        p.check(*p.run(exact=True))
    if form[3] != "bfloat16":
        assert all(torch.equal(a, b) for a, b in zip(p.run(), p.run(exact=True)))
    p = steep(env, form, q8.F32, lambda x: 1.0)
    assert all(torch.equal(a, b) for a, b in zip(p.run(), p.run(exact=True)))


def test_exact_split(env, monkeypatch):  # noqa: F811
    torch, L = env
    monkeypatch.setitem(test_gpu_attn8.WEIGHT, "bfloat16", TWO)
    for new, heads, group in ((1, 4, 4), (70, 1, 4)):
        p = Problem(torch, L, np.random.default_rng(5), [new], [9000], heads=heads, group=group, dim=128, page=64)
        work = torch.empty(L.ds_attn8_work(p.q, p.cache, p.chunk, exact=True), dtype=torch.uint8, device="cuda")
        assert work.numel() > 0
        out, lse = p.run(exact=True, work=work)
        p.check(out, lse, rows={(t, h) for t in (0, new - 1) for h in (0, heads * group - 1)})
        again = p.run(exact=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
