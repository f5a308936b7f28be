"""How far the paged cache's entry points go, on the host: the largest table, and the size of a workspace."""
import pytest

from tests.test_kv_abi import _append, _attn

MOST = (1 << 31) - (1 << 23)                                       # positions of a table


@pytest.mark.parametrize("call", [_append, _attn])
@pytest.mark.parametrize("page", [16, 4096, 65536])
def test_largest_table(call, page):
    """The kernels look some thousand positions past a sequence's end before they cut the position to the end, in 32 bits."""
    none = dict(tokens=0)                                          # nothing is launched
    for width, want in ((MOST // page, 0), (MOST // page + 1, -3), (((1 << 31) - 1) // page, -3)):
        assert call(c=dict(page_size=page), b=dict(table_width=width, table_ld=width, **none)) == want, width
