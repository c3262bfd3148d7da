"""What the 8-bit entry points refuse, before anything is launched (no device needed)."""
import ctypes as C

import pytest

from paper_2406_20037_amd import _lib as L

P = 1 << 20      # a stand-in for a device address; nothing below launches


def q8(rows=4, cols=200, ld=208, sld=2, data=P, scale=P, fmt=0, kind=0, block=1, res=0):
    return L.ds_q8(data, scale, rows, cols, ld, sld, fmt, kind, block, res)


def addr(m):
    return C.addressof(m) if m is not None else None


def quantize(row, col=None, x=P, t=0, rows=4, cols=200, ldx=200):
    return L.lib.ds_q8_quantize(x, t, rows, cols, ldx, addr(row), addr(col), None)


def matmul(a, b, c=P, t=0, ldc=4):
    return L.lib.ds_q8_matmul(addr(a), addr(b), c, t, ldc, None)


BAD = [dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(ld=192), dict(ld=204), dict(ld=1 << 24),
       dict(sld=1), dict(data=None), dict(scale=None), dict(data=P + 8), dict(fmt=2), dict(kind=2),
       dict(block=64), dict(block=0), dict(res=1), dict(kind=1, scale=P + 2)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_bad_matrices(bad):
    assert quantize(q8(**bad)) == L.DS_EINVAL
    assert L.lib.ds_last_error()
    assert matmul(q8(**bad), q8()) == L.DS_EINVAL
    assert matmul(q8(), q8(**bad)) == L.DS_EINVAL


def test_quantize_refusals():
    assert quantize(None) == L.DS_EINVAL
    assert quantize(q8(), t=3) == L.DS_EINVAL
    assert quantize(q8(), x=None) == L.DS_EINVAL
    assert quantize(q8(), x=P + 2) == L.DS_EINVAL
    assert quantize(q8(), ldx=199) == L.DS_EINVAL
    assert quantize(q8(), rows=5) == L.DS_EINVAL
    assert quantize(q8(), q8()) == L.DS_EINVAL                                    # col is cols x rows
    assert quantize(q8(block=128), q8(200, 4, 16, 1)) == L.DS_EINVAL              # squares in one only
    assert quantize(q8(0, 200), rows=0) == L.DS_OK                                # nothing to do


def test_matmul_refusals():
    assert matmul(None, q8()) == L.DS_EINVAL
    assert matmul(q8(), q8(cols=199)) == L.DS_EINVAL
    assert matmul(q8(), q8(kind=1)) == L.DS_EINVAL
    assert matmul(q8(), q8(), ldc=3) == L.DS_EINVAL
    assert matmul(q8(), q8(), c=None) == L.DS_EINVAL
    assert matmul(q8(), q8(), c=P + 1, t=1) == L.DS_EINVAL
    assert matmul(q8(), q8(), t=-1) == L.DS_EINVAL
    assert matmul(q8(0, 200), q8()) == L.DS_OK


def test_swiglu_refusals():
    def call(h=q8(4, 200), saved=None, hidden=200, up=256, ldg=456, gu=P, t=0, rows=4):
        return L.lib.ds_swiglu8(gu, t, rows, hidden, up, ldg, addr(h), addr(saved), None)
    assert call(up=200) == L.DS_EINVAL and call(up=128) == L.DS_EINVAL
    assert call(ldg=455) == L.DS_EINVAL and call(gu=None) == L.DS_EINVAL
    assert call(h=None) == L.DS_EINVAL and call(h=q8(4, 199)) == L.DS_EINVAL
    assert call(h=q8(4, 200, block=128)) == L.DS_EINVAL
    assert call(saved=q8(4, 456, 464, 3)) == L.DS_EINVAL                          # four blocks
    assert call(saved=q8(4, 455, 464, 4)) == L.DS_EINVAL
    assert call(hidden=-1) == L.DS_EINVAL
    assert call(h=q8(0, 200), rows=0) == L.DS_OK


def test_swiglu_grad_refusals():
    s = q8(4, 456, 464, 4)

    def call(saved=s, dh=P, t=0, hidden=200, up=256, ldh=200, dgu=q8(4, 456, 464, 4), dgu_t=None, h_t=None):
        return L.lib.ds_swiglu8_grad(addr(saved), dh, t, hidden, up, ldh, addr(dgu), addr(dgu_t), addr(h_t),
                                     None)
    assert call(saved=None) == L.DS_EINVAL and call(dgu=None) == L.DS_EINVAL
    assert call(dh=None) == L.DS_EINVAL and call(ldh=199) == L.DS_EINVAL
    assert call(up=200) == L.DS_EINVAL and call(saved=q8(4, 455, 464, 4)) == L.DS_EINVAL
    assert call(dgu_t=q8(4, 456, 464, 4)) == L.DS_EINVAL
    assert call(h_t=q8(200, 5, 16, 1)) == L.DS_EINVAL
    assert call(dgu=q8(4, 456, 464, 4, block=128)) == L.DS_EINVAL
    assert call(saved=q8(0, 456, 464, 4), dgu=q8(0, 456, 464, 4)) == L.DS_OK


def test_python_refusals():
    torch = pytest.importorskip("torch")
    f8, s8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    data = torch.zeros(4, 208, dtype=torch.uint8).view(f8)
    scale = torch.zeros(4, 2, dtype=torch.uint8).view(s8)
    m = L.Q8.of(data[:, :200], scale)
    assert (m.rows, m.cols, m._c.ld, m._c.scale_ld) == (4, 200, 208, 2)
    with pytest.raises(ValueError):
        L.Q8.of(data, scale[:3])
    with pytest.raises(ValueError):
        L.Q8.of(data, scale, block_rows=64)
    with pytest.raises(ValueError):
        L.Q8.of(data.t(), scale)
    with pytest.raises(TypeError):
        L.Q8.of(data.view(torch.uint8), scale)
    with pytest.raises(TypeError):
        L.Q8.of(data, torch.zeros(4, 2, dtype=torch.float64))
    with pytest.raises(ValueError):
        L.ds_q8_matmul(m, m, torch.zeros(3, 4))
    with pytest.raises(TypeError):
        L.ds_q8_matmul(m, m, torch.zeros(4, 4, dtype=torch.float64))
    odd = L.Q8.of(torch.zeros(4, 200, dtype=torch.uint8).view(f8), scale)          # rows 200 bytes apart
    assert matmul(odd._c, odd._c) == L.DS_EINVAL
