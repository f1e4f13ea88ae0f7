"""Limits of the paged cache's entries that are checked on the host (no GPU needed)."""
import pytest

from test_paged_cpu import CAPACITY, INVALID, UNSUPPORTED, append, attn, chunk, kv, lib, read  # noqa: F401


@pytest.mark.parametrize("scale,code", [(2.0**127, INVALID), (-2.0**127, INVALID), (3.4e38, INVALID), (2.0**127 * (1 - 2.0**-24), 0),
                                        (-1.7e38, 0), (0.0, 0)])
def test_scales(lib, scale, code):  # noqa: F811
    # no rows: a call that is accepted launches nothing
    assert attn(lib, kv(), chunk(n_rows=0), scale=scale) == code
