"""Strides of an 8-bit cache that no memory holds: refused before 64 bits cut what is computed from them.  Nothing is launched, so no GPU is needed."""
import pytest

from tests.test_kv8_refusals import attend, lib, load, refused, store  # noqa: F401 (lib: a fixture)


@pytest.mark.parametrize("change", [dict(stride_codes=1 << 59), dict(stride_codes=1 << 61), dict(stride_codes=(1 << 63) - 16), dict(stride_scales=1 << 58),
                                    dict(stride_scales=1 << 61), dict(stride_scales=(1 << 63) - 2)])
def test_units_further_apart_than_any_memory(lib, change):
    # four units 2^61 bytes apart: the offset of the last one and the span of all are more than 2^62, and at 2^62 and beyond their sums are negative
    for call in (attend, store, load):
        refused(lib, call(lib, **change), "apart")
