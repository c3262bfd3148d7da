"""The flag of exact sums among the types that the 8-bit entry points take (no device needed)."""
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
