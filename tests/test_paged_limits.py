"""Limits of the paged cache's entries that are checked on the host (no GPU needed)."""
import pytest

from test_paged_cpu import CAPACITY, INVALID, UNSUPPORTED, append, attn, chunk, kv, lib, read  # noqa: F401


@pytest.mark.parametrize("scale,code", [(2.0**127, INVALID), (-2.0**127, INVALID), (3.4e38, INVALID), (2.0**127 * (1 - 2.0**-24), 0),
                                        (-1.7e38, 0), (0.0, 0)])
def test_scales(lib, scale, code):  # noqa: F811
    # no rows: a call that is accepted launches nothing
    assert attn(lib, kv(), chunk(n_rows=0), scale=scale) == code


@pytest.mark.parametrize("entry", [append, read, attn])
def test_positions_up_to_the_end_of_32_bits(lib, entry):  # noqa: F811
    """The kernels count positions up to a few blocks past a sequence's end."""
    wide = dict(n_rows=0, table_stride=32768)
    pool = kv(page_size=65536)
    assert entry(lib, pool, chunk(max_len=2**31 - 1, **wide)) == UNSUPPORTED
    assert entry(lib, pool, chunk(max_len=2**31 - 1023, **wide)) == UNSUPPORTED
    assert entry(lib, pool, chunk(max_len=2**31 - 1024, **wide)) == 0
    assert entry(lib, pool, chunk(max_len=2**31 - 1024, **dict(wide, table_stride=32767))) == CAPACITY
