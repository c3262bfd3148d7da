"""What the entry points around attention refuse, before anything is launched (no device needed)."""
import ctypes as C

import pytest

from paper_2406_20037_amd import _lib as L

P = 1 << 20      # a stand-in for a device address; nothing below launches


def heads(data=P, tokens=4, heads=8, dim=128, ld=1024, head_ld=128, t=2, res=0):
    return L.ds_heads(data, tokens, heads, dim, ld, head_ld, t, res)


def cache(k=P, v=P, ks=P, vs=P, pages=10, stride=2 * 64 * 128, sstride=2 * 64, page=64, heads=2, dim=128, fmt=0,
          kind=0, res=0):
    return L.ds_cache8(k, v, ks, vs, pages, stride, sstride, page, heads, dim, fmt, kind, res)


def chunk(starts=P, lengths=P, table=P, seqs=3, cols=5, ld=5):
    return L.ds_chunk(starts, lengths, table, seqs, cols, ld)


def cfg(scale=0.1, causal=1, res=0, window=0, max_len=0):
    return L.ds_attn8_cfg(scale, causal, res, window, max_len)


def addr(m):
    return C.byref(m) if m is not None else None


def rotary(x, y, turn=128, mode=0, scale=1.0, pos=P, freqs=P):
    return L.lib.ds_rotary(addr(x), pos, freqs, turn, mode, scale, addr(y), None)


def rows(c, n, k, v, name):
    return getattr(L.lib, name)(addr(c), addr(n), addr(k), addr(v), None)


def attn(q=None, c=None, n=None, g=None, out=None, lse=None, work=P, size=1 << 40):
    q, out, c, n, g = q or heads(), out or heads(), c or cache(), n or chunk(), g or cfg()
    return L.lib.ds_attn8(C.byref(q), C.byref(c), C.byref(n), C.byref(g), C.byref(out), lse, work, size, None)


BAD_HEADS = [dict(data=None), dict(data=P + 1), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0),
             dict(heads=65536), dict(dim=0), dict(dim=65537), dict(ld=-1), dict(head_ld=-128), dict(ld=1 << 41),
             dict(t=3), dict(t=-1), dict(res=1)]
OVERLAPS = [dict(head_ld=64), dict(ld=512), dict(ld=0), dict(head_ld=0)]
BAD_CACHE = [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(k=P + 8), dict(v=P + 4),
             dict(kind=1, ks=P + 2), dict(pages=0), dict(pages=1 << 31), dict(stride=2 * 64 * 128 - 16),
             dict(stride=2 * 64 * 128 + 8), dict(sstride=127), dict(page=8), dict(page=40), dict(page=1 << 17),
             dict(heads=0), dict(heads=65536), dict(dim=8), dict(dim=136), dict(dim=272), dict(fmt=2), dict(kind=2),
             dict(res=1), dict(heads=65535, page=65536, stride=1 << 40, sstride=1 << 40), dict(stride=1 << 41)]
BAD_CHUNK = [dict(starts=None), dict(lengths=None), dict(table=None), dict(starts=P + 2), dict(lengths=P + 1),
             dict(table=P + 2), dict(seqs=-1), dict(seqs=(1 << 24) + 1), dict(cols=-1), dict(ld=4),
             dict(cols=1 << 26, ld=1 << 26), dict(ld=1 << 33)]
BAD_CFG = [dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=1e300), dict(causal=2), dict(causal=-1),
           dict(res=1), dict(window=-1), dict(window=5, causal=0), dict(max_len=-1)]


@pytest.mark.parametrize("bad", BAD_HEADS, ids=str)
def test_bad_tensors(bad):
    kv = dict(heads=2, ld=256)
    assert rotary(heads(**bad), heads()) == L.DS_EINVAL
    assert L.lib.ds_last_error()
    assert rotary(heads(), heads(**bad)) == L.DS_EINVAL
    for name in ("ds_cache8_write", "ds_cache8_read"):
        assert rows(cache(), chunk(), heads(**{**kv, **bad}), heads(**kv), name) == L.DS_EINVAL
        assert rows(cache(), chunk(), heads(**kv), heads(**{**kv, **bad}), name) == L.DS_EINVAL
    assert attn(q=heads(**bad)) == L.DS_EINVAL
    assert attn(out=heads(**bad)) == L.DS_EINVAL


@pytest.mark.parametrize("bad", OVERLAPS, ids=str)
def test_outputs_do_not_overlap(bad):
    assert rotary(heads(), heads(**bad)) == L.DS_EINVAL
    assert attn(out=heads(**bad)) == L.DS_EINVAL
    kv = dict(heads=2, ld=256)
    one = {k: v // 4 if k == "ld" else v for k, v in bad.items()}
    assert rows(cache(), chunk(), heads(**kv), heads(**{**kv, **one}), "ds_cache8_read") == L.DS_EINVAL


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches(bad):
    kv = heads(heads=2, ld=256)
    for name in ("ds_cache8_write", "ds_cache8_read"):
        assert rows(cache(**bad), chunk(), kv, kv, name) == L.DS_EINVAL
    assert attn(c=cache(**bad)) == L.DS_EINVAL
    assert rows(None, chunk(), kv, kv, "ds_cache8_write") == L.DS_EINVAL


@pytest.mark.parametrize("bad", BAD_CHUNK, ids=str)
def test_bad_chunks(bad):
    kv = heads(heads=2, ld=256)
    for name in ("ds_cache8_write", "ds_cache8_read"):
        assert rows(cache(), chunk(**bad), kv, kv, name) == L.DS_EINVAL
    assert attn(n=chunk(**bad)) == L.DS_EINVAL
    assert rows(cache(), None, kv, kv, "ds_cache8_write") == L.DS_EINVAL


@pytest.mark.parametrize("bad", BAD_CFG, ids=str)
def test_bad_settings(bad):
    assert attn(g=cfg(**bad)) == L.DS_EINVAL
    n = C.c_int64()
    assert L.lib.ds_attn8_work(addr(heads()), addr(cache()), addr(chunk()), addr(cfg(**bad)), C.byref(n)) == L.DS_EINVAL


def test_rotary_refusals():
    x = heads()
    for bad in (dict(turn=-2), dict(turn=3), dict(turn=130), dict(mode=4), dict(mode=-1), dict(pos=None),
                dict(freqs=None), dict(pos=P + 2), dict(freqs=P + 1), dict(scale=float("inf")),
                dict(scale=float("nan"))):
        assert rotary(x, x, **bad) == L.DS_EINVAL, bad
    assert rotary(None, x) == rotary(x, None) == L.DS_EINVAL
    assert rotary(heads(dim=65536, ld=1 << 20, head_ld=65536), heads(dim=65536, ld=1 << 20, head_ld=65536),
                  turn=4098) == L.DS_EINVAL
    for other in (dict(tokens=5), dict(heads=7), dict(dim=127), dict(t=1)):
        assert rotary(x, heads(**other)) == L.DS_EINVAL, other
    none = heads(data=None, tokens=0)
    assert rotary(none, none) == L.DS_OK
    assert rotary(x, x, turn=0, freqs=None) == L.DS_OK                   # in place, nothing turns


def test_row_refusals():
    kv = dict(heads=2, ld=256)
    for name in ("ds_cache8_write", "ds_cache8_read"):
        for bad in (dict(tokens=5), dict(heads=1), dict(dim=64), dict(t=0)):
            assert rows(cache(), chunk(), heads(**kv), heads(**{**kv, **bad}), name) == L.DS_EINVAL, bad
        assert rows(cache(), chunk(), heads(**{**kv, "heads": 4}), heads(**{**kv, "heads": 4}), name) == L.DS_EINVAL
        none = heads(**{**kv, "tokens": 0, "data": None})
        assert rows(cache(), chunk(), none, none, name) == L.DS_OK
        assert rows(cache(), chunk(None, None, None, 0, 0, 0), heads(**kv), heads(**kv), name) == L.DS_OK


def test_attention_refusals():
    assert attn(q=heads(heads=7), out=heads(heads=7)) == L.DS_EINVAL               # heads that do not share
    assert attn(q=heads(dim=64), out=heads(dim=64)) == L.DS_EINVAL
    for other in (dict(tokens=5), dict(heads=16), dict(dim=64), dict(t=1)):
        assert attn(out=heads(**other)) == L.DS_EINVAL, other
    assert attn(lse=P + 2) == L.DS_EINVAL
    wide = dict(dim=256, ld=2048, head_ld=256, t=0)
    assert attn(q=heads(**wide), out=heads(**wide), c=cache(dim=256, stride=2 * 64 * 256)) == L.DS_EUNSUPPORTED
    none = heads(tokens=0, data=None)
    assert attn(q=none, out=none, work=None, size=0) == L.DS_OK
    assert attn(n=chunk(None, None, None, 0, 0, 0), work=None, size=0) == L.DS_OK


def test_workspace():
    n = C.c_int64()
    one = heads(tokens=3)

    def need(**kw):
        assert L.lib.ds_attn8_work(addr(one), addr(cache()), addr(chunk(**kw)), addr(cfg()), C.byref(n)) == L.DS_OK
        return n.value
    assert need(cols=1) == 0                                                        # nothing to split
    size = need(cols=500, ld=500)
    assert size > 0 and size % 8 == 0
    long = chunk(cols=500, ld=500)
    for work, have in ((None, size), (P, size - 1), (P + 8, size), (P, 0)):
        assert attn(q=one, out=one, n=long, work=work, size=have) == L.DS_EINVAL
        assert b"workspace" in L.lib.ds_last_error()
    assert L.lib.ds_attn8_work(addr(one), addr(cache()), addr(long), addr(cfg()), None) == L.DS_EINVAL


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.ones(4, 2, 16)
    L.Cache8.of(k, k, s, s)
    for bad in ((k.view(torch.uint8), k, s, s), (k, k.view(torch.float8_e5m2), s, s), (k, k, s.half(), s),
                (k, k, s, s.to(torch.float8_e8m0fnu))):
        with pytest.raises(TypeError):
            L.Cache8.of(*bad)
    for bad in ((k, k[:3], s, s), (k, k, s[:, :1], s), (k.transpose(1, 2), k.transpose(1, 2), s, s),
                (k[::2], k[:2], s[:2], s[:2])):
        with pytest.raises(ValueError):
            L.Cache8.of(*bad)
    starts, lengths, table = (torch.zeros(n, dtype=torch.int32) for n in ((3,), (2,), (2, 4)))
    L.Chunk(starts, lengths, table)
    for bad in ((starts.long(), lengths, table), (starts, lengths, table[0]), (starts, lengths.float(), table)):
        with pytest.raises(TypeError):
            L.Chunk(*bad)
    for bad in ((starts[:2], lengths, table), (starts, lengths, table[:1]), (starts, lengths, table.t().contiguous().t())):
        with pytest.raises(ValueError):
            L.Chunk(*bad)
    with pytest.raises(ValueError, match="side by side"):
        L._heads(torch.zeros(2, 3, 8)[..., ::2])
    with pytest.raises(TypeError):
        L._heads(torch.zeros(2, 3, 8, dtype=torch.float64))
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="the host"):
        L.ds_rotary(x, torch.zeros(2, dtype=torch.int32), torch.zeros(4))
    with pytest.raises(ValueError, match="the host"):
        L.ds_attn8(x, L.Cache8.of(k, k, s, s), L.Chunk(starts, lengths, table), x)
    with pytest.raises(ValueError, match="the host"):
        L.ds_cache8_write(L.Cache8.of(k, k, s, s), L.Chunk(starts, lengths, table), x, x)
