"""How the host splits attention over the cache (no device needed: the workspace's size tells)."""
import ctypes as C

from paper_2406_20037_amd import _lib as L
from test_capi_attn8 import cache, cfg, chunk, heads


def size(window=0, max_len=0, tokens=1):
    n = C.c_int64()
    args = heads(tokens=tokens), cache(), chunk(cols=1 << 12, ld=1 << 12, seqs=tokens), cfg(window=window, max_len=max_len)
    assert L.lib.ds_attn8_work(*(C.byref(a) for a in args), C.byref(n)) == L.DS_OK
    return n.value


def test_windows_and_lengths_past_everything():
    """They see what no window and no most length see, up to the largest numbers."""
    assert size() > 0
    for far in (1 << 18, (1 << 31) - 1, 1 << 31, 1 << 40, (1 << 63) - 65, (1 << 63) - 1):
        assert size(window=far) == size() == size(max_len=far)


def test_a_window_bounds_the_split():
    """A short window leaves few splits, whatever the sequences' length."""
    assert size(window=100) <= size(window=4000) <= size()
    assert size(window=1) < size()
