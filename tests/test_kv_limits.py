"""How far the paged cache's entry points go, on the host: the largest table, and the size of a workspace."""
import pytest

from paper_2603_08185_amd import binding as serq
from tests.test_kv_abi import _append, _attn

MOST = (1 << 31) - (1 << 23)                                       # positions of a table


@pytest.mark.parametrize("call", [_append, _attn])
@pytest.mark.parametrize("page", [16, 4096, 65536])
def test_largest_table(call, page):
    """The kernels look some thousand positions past a sequence's end before they cut the position to the end, in 32 bits."""
    none = dict(tokens=0)                                          # nothing is launched
    for width, want in ((MOST // page, 0), (MOST // page + 1, -3), (((1 << 31) - 1) // page, -3)):
        assert call(c=dict(page_size=page), b=dict(table_width=width, table_ld=width, **none)) == want, width


def _size(tokens, seqs, max_q, max_kv, heads=(32, 8, 128)):
    return serq.lib().serq_paged_attn_workspace_bytes(tokens, seqs, max_q, max_kv, *heads)


@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 32, 64), (8, 1, 128), (32, 1, 128), (64, 1, 64), (40, 2, 128), (14, 2, 64)])
def test_a_workspace_serves_every_smaller_call(heads):
    """Sized once for the largest step, it has room for what a step of fewer tokens, sequences or keys takes."""
    steps = [(t, s, q, k) for t in (0, 1, 8, 48, 512, 8192, 1 << 17) for s in (0, 1, 7, 48, 512) for q in (0, 1, 5, 33, 512, 8192) if q <= t
             for k in (0, 1, 200, 1000, 16000, 131072, 1 << 24)]
    size = {x: _size(*x, heads) for x in steps}
    for a, x in enumerate(steps):
        assert size[x] > 0
        for i in range(4):                                         # against the next larger value of each
            more = sorted({y[i] for y in steps if all(y[j] == x[j] for j in range(4) if j != i) and y[i] > x[i]})
            if more:
                y = (*x[:i], more[0], *x[i + 1:])
                assert size[x] <= size[y], (x, y)


def test_a_workspace_is_no_larger_than_what_can_be_used():
    """Tickets, two slots for each workgroup of the kernel for few rows, 46 MiB for the slices of the kernel for many."""
    for x in ((1, 1, 1, 131072), (48, 48, 1, 131072), (8192, 64, 8192, 131072), (1 << 22, 16384, 1 << 22, 1 << 30)):
        few = 32768 + 2 * 512 * (16 if x[2] * 4 <= 16 else 32) * 130 * 4
        assert _size(*x) <= few + (0 if x[2] * 4 <= 32 else 46 << 20), x
    assert _size(1, 1, 1, 200) <= 32768 + 2 * 16 * 16 * 130 * 4    # (and a short sequence has few parts)
