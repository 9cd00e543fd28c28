"""Strides of the embedding calls whose extents do not fit 64 bits (no kernel is launched, so no GPU is needed)."""
import pytest

from test_more_operators_host import SHAPE, embed_call, rdk  # noqa: F401


@pytest.mark.parametrize("which", ["forward", "grad"])
@pytest.mark.parametrize("tt", [1, 2])
def test_tables_beyond_any_memory_are_refused(rdk, which, tt):  # noqa: F811
    """2^29 rows at a stride of 2^34: 2^65 bytes of fp32, 2^64 of bf16; lower ones that lie over nothing once they are cut to 64 bits; each wherever the table begins."""
    for V, ldt in ((1 << 29, 1 << 34), ((1 << 29) - 1, (1 << 34) - 7), ((1 << 28) + 1, 1 << 34), ((1 << 29), (1 << 33) + 64), (1 << 29, (1 << 32) + 16)):
        for table in (0x200000, 0x7F0000000000):
            assert embed_call(rdk, which, V=V, ldt=ldt, tt=tt, table=table) == SHAPE, (V, ldt, table)
