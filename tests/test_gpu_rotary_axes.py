"""Rotary positions with several axes, their table and gradient, against the definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2407_13885_amd as attnw
from byte_util import axis_map
from gpu_util import DT, TORCH_DT, require_gpu
from paged_util import EPS, within
from test_gpu_rotary import bound_of

pytestmark = pytest.mark.gpu

SECTIONS, TURNS, HALVES, PAIRS = attnw.ATTNW_SECTIONS, attnw.ATTNW_TURNS, attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def table_of(rows, pairs, order, fresh, base=10000.0, gain=1.0, factor=1.0, low=0.0, high=0.0, original=0.0):
    axis, index = axis_map(pairs, order)
    n = len(axis)
    f = base ** -np.array([i / pairs[a] if fresh else j / n for j, (a, i) in enumerate(zip(axis, index))])
    turns = original * f / (2 * math.pi)
    with np.errstate(invalid="ignore"):
        k = np.where(turns >= high, 1.0, np.where(turns <= low, 0.0, (turns - low) / (high - low)))
    angle = np.arange(rows)[:, None] * (f * (k + (1 - k) / factor))
    return torch.from_numpy(gain * np.concatenate([np.cos(angle), np.sin(angle)], 1))


@pytest.mark.parametrize("order", [SECTIONS, TURNS])
@pytest.mark.parametrize("rows,pairs,fresh,scaling", [
    (1, [1], 0, {}), (500, [16, 24, 24], 0, dict(base=500000.0)), (777, [16, 16], 1, {}), (300, [3, 1, 7, 2], 1, dict(gain=1.25)),
    (2000, [40, 44, 44], 1, dict(factor=8.0, low=1.0, high=4.0, original=1024.0)), (100001, [8, 4], 0, dict(factor=2.0, low=math.inf, high=math.inf)),
])
def test_table(order, rows, pairs, fresh, scaling):
    rot = 2 * sum(pairs)
    table = torch.full((rows, rot), 7.0, device="cuda")
    attnw.attnw_rotary_axes_table(table, attnw.AttnwAxes(pairs, order, fresh), rows, rot, **scaling)
    torch.cuda.synchronize()
    gain = scaling.get("gain", 1.0)
    # one rounding of each side; an angle is good to a few 2^-52 of itself in 64 bits, on either side
    within(table, table_of(rows, pairs, order, fresh, **scaling), torch.full((rows, rot), gain * (EPS + 16 * rows * 2.0 ** -52)) + gain * EPS, "table")


def test_table_of_one_run_of_frequencies_is_that_of_one_axis():
    one, other = torch.empty((3000, 96), device="cuda"), torch.empty((3000, 96), device="cuda")
    attnw.attnw_rotary_table(one, 3000, 96, base=500000.0)
    attnw.attnw_rotary_axes_table(other, attnw.AttnwAxes([20, 20, 8], TURNS), 3000, 96, base=500000.0)
    within(other, one.cpu().double(), torch.full((3000, 96), EPS + 16 * 3000 * 2.0 ** -52), "table")


def turned(x, table, positions, pairs, order, layout, inverse=False):
    """x [T][heads][d] in 64 bits, pair by pair."""
    y = x.double().clone()
    half = len(axis_map(pairs, order)[0])
    for j, a in enumerate(axis_map(pairs, order)[0]):
        row = table[positions[a].long()].double()
        c, s = row[:, j, None], row[:, half + j, None] * (-1.0 if inverse else 1.0)
        p, q = (j, half + j) if layout == HALVES else (2 * j, 2 * j + 1)
        y[..., p], y[..., q] = x[..., p].double() * c - x[..., q].double() * s, x[..., q].double() * c + x[..., p].double() * s
    return y


# tokens, heads, d, pairs: sections that vectors do and do not fall into, whole heads and parts, one axis to four
SHAPES = [(1, 1, 64, [32]), (37, 3, 128, [16, 24, 24]), (300, 2, 128, [64]), (33, 5, 80, [14, 13, 13]), (70, 4, 64, [5, 3, 7, 1]), (9, 4, 256, [32, 96]),
          (1000, 1, 64, [1, 1, 1]), (3, 2, 72, [12, 12, 12]), (129, 20, 48, [2, 6]), (5, 3, 50, [7, 4]), (2, 1, 16, [4, 4]),
          (33, 3, 36, [4, 5]), (21, 2, 36, [6, 4]), (11, 5, 26, [5, 4, 4]), (301, 16, 72, [1, 3, 2, 3]), (71, 7, 44, [10, 2])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [HALVES, PAIRS])
@pytest.mark.parametrize("order", [SECTIONS, TURNS])
@pytest.mark.parametrize("tokens,heads,d,pairs", SHAPES, ids=[str(s) for s in SHAPES])
def test_rotary_axes(dtype, layout, order, tokens, heads, d, pairs):
    g = torch.Generator().manual_seed(tokens + d)
    rows, t, rot = 500, TORCH_DT[dtype], 2 * sum(pairs)
    table = table_of(rows, pairs, order, 0).float()
    positions = torch.randint(0, rows, (len(pairs), tokens), generator=g, dtype=torch.int32)
    pad = 24 if tokens % 2 else 3                 # (rows on and off the 16-byte boundaries)
    x = torch.randn((tokens, heads * d + pad), generator=g).to(t)
    dev, table_dev, pos_dev, axes = x.cuda(), table.cuda(), positions.cuda(), attnw.AttnwAxes(pairs, order)
    heads_of = x[:, :heads * d].view(tokens, heads, d)
    for inverse in (0, 1):
        y = torch.full((tokens, heads * d + 8), 7.0, dtype=t, device="cuda")
        attnw.attnw_rotary_axes(dev, y, table_dev, pos_dev, axes, tokens, heads, d, rot, rows, heads * d + pad, heads * d + 8, layout, inverse, DT[dtype])
        torch.cuda.synchronize()
        assert bool((y[:, heads * d:] == 7.0).all())
        got = y[:, :heads * d].reshape(tokens, heads, d)
        within(got, turned(heads_of, table, positions, pairs, order, layout, inverse), bound_of(heads_of, dtype), "rotary_axes")
        assert torch.equal(got[..., rot:].cpu(), heads_of[..., rot:])
    attnw.attnw_rotary_axes(dev, dev, table_dev, pos_dev, axes, tokens, heads, d, rot, rows, heads * d + pad, heads * d + pad, layout, 1, DT[dtype])   # in place
    torch.cuda.synchronize()
    assert torch.equal(dev[:, :heads * d].reshape(tokens, heads, d), got) and torch.equal(dev[:, heads * d:].cpu(), x[:, heads * d:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_axis_is_attnw_rotary(dtype):
    g = torch.Generator().manual_seed(5)
    x = torch.randn((77, 6 * 64), generator=g).to(TORCH_DT[dtype]).cuda()
    table = torch.empty((100, 48), device="cuda")
    attnw.attnw_rotary_table(table, 100, 48)
    positions = torch.randint(0, 100, (77,), generator=g, dtype=torch.int32).cuda()
    a, b, c = (torch.empty_like(x) for _ in range(3))
    attnw.attnw_rotary(x, a, table, positions, 77, 6, 64, 48, 100, 384, 384, HALVES, 0, DT[dtype])
    attnw.attnw_rotary_axes(x, b, table, positions, attnw.AttnwAxes([24]), 77, 6, 64, 48, 100, 384, 384, HALVES, 0, DT[dtype])
    attnw.attnw_rotary_axes(x, c, table, positions.repeat(3), attnw.AttnwAxes([9, 9, 6], TURNS), 77, 6, 64, 48, 100, 384, 384, HALVES, 0, DT[dtype])
    assert torch.equal(a, b) and torch.equal(a, c)


def test_positions_that_the_table_does_not_have():
    """An axis whose row is missing spoils its own columns."""
    rows, pairs = 10, [4, 2, 2]
    positions = torch.tensor([[0, 10, 3], [1, 2, -1], [9, 9, 2 ** 31 - 1]], dtype=torch.int32)
    table = table_of(rows, pairs, SECTIONS, 0).float()
    x = torch.randn((3, 2, 24), generator=torch.Generator().manual_seed(1))
    for layout in (HALVES, PAIRS):
        y = torch.empty((3, 2, 24), device="cuda")
        attnw.attnw_rotary_axes(x.cuda(), y, table.cuda(), positions.cuda(), attnw.AttnwAxes(pairs), 3, 2, 24, 16, rows, 48, 48, layout, 0, attnw.ATTNW_F32)
        torch.cuda.synchronize()
        nan = torch.zeros((3, 24), dtype=torch.bool)
        for t, lost in ((1, range(0, 4)), (2, range(4, 8))):
            for j in lost:
                nan[t, [j, 8 + j] if layout == HALVES else [2 * j, 2 * j + 1]] = True
        assert torch.equal(y.isnan().cpu(), nan[:, None].expand(3, 2, 24))


def test_gradient_by_differences():
    """d/dx of sum(w * turned(x)) is the transposed map of w."""
    pairs, rows, d, T, heads = [3, 5, 4], 64, 32, 6, 2
    g = torch.Generator().manual_seed(2)
    table = table_of(rows, pairs, TURNS, 1, gain=1.5).float().cuda()
    positions = torch.randint(0, rows, (3, T), generator=g, dtype=torch.int32).cuda()
    x, w = (torch.randn((T, heads, d), generator=g).cuda() for _ in range(2))

    def run(v, inverse):
        y = torch.empty_like(v)
        attnw.attnw_rotary_axes(v, y, table, positions, attnw.AttnwAxes(pairs, TURNS), T, heads, d, 24, rows, heads * d, heads * d, PAIRS, inverse, attnw.ATTNW_F32)
        torch.cuda.synchronize()
        return y.double()
    grad = run(w, 1)
    for t, h, c in ((0, 0, 0), (1, 1, 7), (3, 0, 23), (5, 1, 12), (2, 0, 30)):
        step = torch.zeros_like(x)
        step[t, h, c] = 0.5
        high, low = run(x + step, 0), run(x - step, 0)
        # the map is linear: the difference is the derivative but for roundings of either side (numbers up to 8, 3 of them each)
        assert abs(float((w.double() * (high - low)).sum()) - float(grad[t, h, c])) <= 2 * 3 * 2.0 ** -24 * 8 * float(w.abs().sum())


def test_long_rows_and_streams():
    """Strides past 2^31 elements from the first token to the last; another stream than the tensors' own."""
    d, stride, T = 16, 1 << 26, 34
    x = torch.zeros(stride * (T - 1) + d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(3)
    rows = torch.randn((T, 1, d), generator=g).to(torch.bfloat16)
    for t in range(T):
        x[t * stride:t * stride + d] = rows[t, 0].cuda()
    table = table_of(40, [3, 5], SECTIONS, 0).float()
    positions = torch.randint(0, 40, (2, T), generator=g, dtype=torch.int32)
    table_dev, pos_dev = table.cuda(), positions.cuda()
    y = torch.empty((T, 1, d), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    attnw.attnw_rotary_axes(x, y, table_dev, pos_dev, attnw.AttnwAxes([3, 5]), T, 1, d, 16, 40, stride, d, HALVES, 0, attnw.ATTNW_BF16, side)
    side.synchronize()
    within(y, turned(rows, table, positions, [3, 5], SECTIONS, HALVES), bound_of(rows, "bf16"), "far rows")
