"""DS_EXACT_SUMS in the type of attention's queries, and nowhere else (no device needed)."""
import ctypes as C

import pytest

from paper_2406_20037_amd import _lib as L
from test_capi_attn8 import addr, attn, cache, cfg, chunk, heads, rotary, rows


@pytest.mark.parametrize("t", [0, 1, 2])
def test_queries_take_it(t):
    q, plain, none = heads(t=t + L.DS_EXACT_SUMS), heads(t=t), dict(tokens=0, data=None)
    assert attn(q=heads(t=t + L.DS_EXACT_SUMS, **none), out=heads(t=t, **none), work=None, size=0) == L.DS_OK
    n, m = C.c_int64(), C.c_int64()
    for x, size in ((q, n), (plain, m)):
        assert L.lib.ds_attn8_work(addr(x), addr(cache()), addr(chunk(cols=500, ld=500)), addr(cfg()), C.byref(size)) == L.DS_OK
    assert n.value == m.value > 0
    assert attn(q=q, out=heads(t=(t + 1) % 3)) == L.DS_EINVAL


def test_nothing_else_does():
    e = L.DS_EXACT_SUMS
    assert attn(q=heads(t=2 + e), out=heads(t=2 + e)) == attn(out=heads(t=2 + e)) == L.DS_EINVAL
    assert attn(q=heads(t=3 + e)) == attn(q=heads(t=2 + 2 * e)) == L.DS_EINVAL
    assert rotary(heads(t=2 + e), heads(t=2 + e)) == L.DS_EINVAL
    kv = heads(heads=2, ld=256, t=2 + e)
    for name in ("ds_cache8_write", "ds_cache8_read"):
        assert rows(cache(), chunk(), kv, kv, name) == L.DS_EINVAL
    assert L.lib.ds_attn8_work(None, addr(cache()), addr(chunk()), addr(cfg()), C.byref(C.c_int64())) == L.DS_EINVAL
