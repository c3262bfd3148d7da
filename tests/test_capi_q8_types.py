"""The flag of exact sums among the types that the 8-bit entry points take, and matrices whose strides say
nothing (no device needed)."""
import pytest

from paper_2406_20037_amd import _lib as L
from test_capi_q8 import matmul, q8, quantize


@pytest.mark.parametrize("t", [3, 255, -1, 512, 1 << 30])
def test_unknown_types_with_and_without_the_flag(t):
    assert matmul(q8(), q8(), t=t) == L.DS_EINVAL
    assert matmul(q8(), q8(), t=t | L.DS_EXACT_SUMS) == L.DS_EINVAL


def test_the_flag_is_the_products_alone():
    for t in (L.DS_TYPE_F32, L.DS_TYPE_F16, L.DS_TYPE_BF16):
        assert matmul(q8(0, 200), q8(), t=t + L.DS_EXACT_SUMS) == L.DS_OK
        assert quantize(q8(), t=t + L.DS_EXACT_SUMS) == L.DS_EINVAL


@pytest.mark.parametrize("rows", [0, 1])
@pytest.mark.parametrize("apart", [200, 208, 1 << 24])
def test_the_stride_of_a_single_row(rows, apart):
    """One row, or none, of values any distance apart: accepted, as a single row has no next."""
    torch = pytest.importorskip("torch")
    data = torch.zeros(256, dtype=torch.uint8).as_strided((rows, 200), (apart, 1)).view(torch.float8_e4m3fn)
    scale = torch.zeros(8, dtype=torch.uint8).as_strided((rows, 2), (apart, 1)).view(torch.float8_e8m0fnu)
    m = L.Q8.of(data, scale)
    assert (m._c.ld, m._c.scale_ld) == (208, 4)
    # the host's checks alone: a second operand without rows launches nothing
    none = L.Q8(0, 200, device="cpu")
    assert L.lib.ds_q8_matmul(m._p, none._p, None, L.DS_TYPE_F32, 0, None) == L.DS_OK


def test_more_workgroups_than_a_launch_takes():
    """A launch counts its threads in 32 bits: shapes within the limits of a matrix that need more."""
    wide = 0x7ffffe00
    assert quantize(None, q8(wide, 1, 16, 1), rows=1, cols=wide, ldx=wide) == L.DS_EUNSUPPORTED
    assert matmul(q8(1, 4096, 4096, 32), q8(wide, 4096, 4096, 32), ldc=wide) == L.DS_EUNSUPPORTED
    assert b"workgroups" in L.lib.ds_last_error()
