"""Rows of tokens that are longer than what the threads of a workgroup turn at once (rotary positions with several axes, appending to a cache in 8 bits): several
rounds of a workgroup, and several workgroups a token where there are few tokens."""
import pytest
import torch

import paper_2407_13885_amd as attnw
from byte_util import Problem8
from gpu_util import DT, TORCH_DT, require_gpu
from paged_util import within
from test_gpu_byte_append import check, new_rows, run
from test_gpu_rotary import bound_of
from test_gpu_rotary_axes import table_of, turned

pytestmark = pytest.mark.gpu

SECTIONS, TURNS, HALVES, PAIRS = attnw.ATTNW_SECTIONS, attnw.ATTNW_TURNS, attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


# (units of a token: 512 and 1024 of 16 bytes; 2 x 8 times that where turned columns fall into single elements)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [HALVES, PAIRS])
@pytest.mark.parametrize("heads,d,rot,pairs", [(32, 128, 128, [16, 24, 24]), (64, 128, 128, None), (33, 256, 6, [1, 1, 1]), (40, 128, 98, None), (50, 112, 60, [7, 13, 10])])
@pytest.mark.parametrize("tokens", [1, 3, 60, 530])
def test_append(dtype, layout, heads, d, rot, pairs, tokens):
    p = Problem8(dtype, [(tokens, tokens + 40)], heads, 1, d, 16, 8, seed=heads).on_gpu()
    positions = None if pairs is None else torch.randint(0, 600, (3, tokens), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    R, q, want_R, want = run(p, new_rows(p), rot, layout, pairs, TURNS, positions, rows=600)
    check(p, want)
    within(R, want_R.double(), 2 * bound_of(q, dtype), "R")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [HALVES, PAIRS])
@pytest.mark.parametrize("order", [SECTIONS, TURNS])
@pytest.mark.parametrize("heads,d,pairs", [(48, 128, [22, 21, 21]), (40, 256, [50, 14, 64]), (70, 72, [3, 3, 3]), (130, 64, [9, 9, 14])])
@pytest.mark.parametrize("tokens", [1, 5, 700])
def test_rotary_axes(dtype, layout, order, heads, d, pairs, tokens):
    g = torch.Generator().manual_seed(tokens + d)
    rows, rot, wide = 500, 2 * sum(pairs), heads * d
    table = table_of(rows, pairs, order, 0).float()
    positions = torch.randint(0, rows, (3, tokens), generator=g, dtype=torch.int32)
    x = torch.randn((tokens, heads, d), generator=g).to(TORCH_DT[dtype])
    dev, table_dev, pos_dev, axes = x.cuda(), table.cuda(), positions.cuda(), attnw.AttnwAxes(pairs, order)
    y = torch.full_like(dev, 7.0)
    for inverse in (1, 0):
        attnw.attnw_rotary_axes(dev, y, table_dev, pos_dev, axes, tokens, heads, d, rot, rows, wide, wide, layout, inverse, DT[dtype])
        torch.cuda.synchronize()
        within(y, turned(x, table, positions, pairs, order, layout, bool(inverse)), bound_of(x, dtype), "rotary_axes")
    attnw.attnw_rotary_axes(dev, dev, table_dev, pos_dev, axes, tokens, heads, d, rot, rows, wide, wide, layout, 0, DT[dtype])   # in place
    torch.cuda.synchronize()
    assert torch.equal(dev, y)
