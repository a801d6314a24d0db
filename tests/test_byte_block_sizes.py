"""The longest blocks of slots that appending to a paged cache in 8 bits takes: 2^30 elements of a head (its units are counted in 32 bits)."""
import pytest

from test_api_cpu import E_ALIGN, E_UNSUP
from test_byte_api import Q, append, attend, cache


# (Q off its alignment: what is not refused for its sizes is refused for that, and nothing is launched)
@pytest.mark.parametrize("slots,block,d,want", [(1 << 23, 1 << 23, 256, E_UNSUP), (1 << 23, 1 << 22, 256, E_ALIGN), ((1 << 22) + 2, (1 << 22) + 2, 256, E_UNSUP),
                                                (1 << 26, 1 << 26, 32, E_UNSUP), (1 << 26, 1 << 25, 32, E_ALIGN), (1 << 27, 1 << 27, 16, E_UNSUP), (1 << 26, 1 << 26, 16, E_ALIGN),
                                                (16777215, 16777215, 64, E_ALIGN), (16777217, 16777217, 64, E_UNSUP)])
def test_long_blocks(slots, block, d, want):
    c = cache(pages=1, max_pages=1, batch=1, page_size=slots, block=block, kv_heads=1, d=d)
    for rot in (0, 2, 16):
        assert append(c, q=Q + 2, tokens=slots, heads=0, rot=rot, qs=0, kvs=d) == want
    assert attend(c, q=Q + 2, tokens=1, heads=1, stride=d) == E_ALIGN         # (attention counts no units)
