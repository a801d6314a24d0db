"""NaN of any bits among rows that are appended to a paged cache in 8 bits: they become NaN and leave their block its scale, quiet or signalling, wherever in a row they are."""
import pytest
import torch

import paper_2407_13885_amd as attnw
from byte_util import Problem8, is_nan, same_bytes
from gpu_util import require_gpu
from test_gpu_byte_append import check, new_rows, run

pytestmark = pytest.mark.gpu

# the shortest signalling NaN, one of all bits but the first of the mantissa, and a quiet one
BITS = {"bf16": [0x7f81, 0xffbf - 0x10000, 0x7fc0], "f32": [0x7f800001, 0xffbfffff - 0x100000000, 0x7fc00000]}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", range(3), ids=["signalling", "signalling, negative", "quiet"])
@pytest.mark.parametrize("layout", [attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS])
@pytest.mark.parametrize("rot", [0, 2, 16])
@pytest.mark.parametrize("block", [4, 16])
def test_a_row_with_a_nan(dtype, which, layout, rot, block):
    """A block for every column: its largest element in one, and NaN behind it (in the block's last row in front of it)."""
    d, slots = 32, 64 * block
    p = Problem8(dtype, [(slots, slots)], 1, 1, d, block, block, seed=rot).on_gpu()
    x = new_rows(p, 3, spread=0.0)
    bits = x.view(torch.int16 if dtype == "bf16" else torch.int32)
    for b in range(64):
        row, column, back = b * block + (b % block), b % 32, b >= 32
        other = (column + 1 + b % 7) % 32
        for first in (d, 2 * d):                  # keys, values
            x[row, first + column] = 3000.0
            bits[row - 1 if back and row % block else row, first + other] = BITS[dtype][which]
    R, q, _, want = run(p, x, rot, layout, rows=slots + 1)
    check(p, want)
    for name in "KV":                             # (and there is one in every block)
        assert bool(is_nan(p.dev[name + "8"].cpu()[p.table[0].long()]).flatten(1).any(1).all())


def test_nothing_but_nan():
    """A block of signalling NaN alone has the least scale."""
    p = Problem8("bf16", [(8, 8)], 1, 1, 32, 8, 8).on_gpu()
    x = new_rows(p)
    x.view(torch.int16)[:, 32:] = 0x7f81
    run(p, x, 0)
    page = int(p.table[0, 0])
    for name in "KV":
        assert int(p.dev[name + "_scales"][page, 0, 0]) == 127 - 117
        same_bytes(p.dev[name + "8"][page], torch.full((1, 8, 32), 0x7f, dtype=torch.uint8), name)
