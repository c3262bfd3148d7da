"""Outputs whose rows overlap at strides where tokens times the distance between them is past 64 bits (no device needed)."""
import pytest

from paper_2406_20037_amd import _lib as L
from test_capi_attn8 import attn, cache, chunk, heads, rotary, rows

FAR = dict(tokens=(1 << 24) + 1, ld=1 << 40, head_ld=1 << 40)      # the next head's row is the next token's


@pytest.mark.parametrize("tokens", [(1 << 24) + 1, (1 << 23) + 1, (1 << 25) + 3])
def test_far_strides(tokens):
    far = dict(FAR, tokens=tokens)
    assert rotary(heads(**far), heads(**far), turn=0, freqs=None) == L.DS_EINVAL
    assert b"overlap" in L.lib.ds_last_error()
    assert attn(q=heads(**far), out=heads(**far), size=0) == L.DS_EINVAL
    assert b"overlap" in L.lib.ds_last_error()
    kv = heads(**dict(far, heads=2))
    assert rows(cache(), chunk(None, None, None, 0, 0, 0), kv, kv, "ds_cache8_read") == L.DS_EINVAL
