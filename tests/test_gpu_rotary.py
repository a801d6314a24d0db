"""Rotary positions, their table and gradient, and appending to a paged cache, against the definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2407_13885_amd as attnw
from gpu_util import DT, TORCH_DT, require_gpu
from paged_util import EPS, Problem, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def frequencies(rot, base, factor=1.0, low=0.0, high=0.0, original=0.0):
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    turns = original * f / (2 * math.pi)
    with np.errstate(invalid="ignore"):
        k = np.where(turns >= high, 1.0, np.where(turns <= low, 0.0, (turns - low) / (high - low)))
    return f * (k + (1 - k) / factor)


def table_of(rows, rot, base=10000.0, gain=1.0, **scaling):
    angle = np.arange(rows)[:, None] * frequencies(rot, base, **scaling)
    return torch.from_numpy(gain * np.concatenate([np.cos(angle), np.sin(angle)], 1)).float()


@pytest.mark.parametrize("rows,rot,scaling", [
    (1, 2, {}), (7, 64, {}), (5000, 128, dict(base=500000.0)), (1500, 96, dict(factor=4.0, low=math.inf, high=math.inf)),
    (3000, 128, dict(factor=8.0, low=1.0, high=4.0, original=8192.0, base=500000.0, gain=1.1)), (200001, 16, dict(factor=2.5, low=1.0, high=32.0, original=4096.0)),
])
def test_table(rows, rot, scaling):
    table = torch.full((rows, rot), 7.0, device="cuda")
    attnw.attnw_rotary_table(table, rows, rot, **scaling)
    torch.cuda.synchronize()
    gain = scaling.get("gain", 1.0)
    # one rounding; angles up to 2 * 10^5 are good to 2^-52 of that in 64 bits, on either side
    bound = torch.full((rows, rot), gain * (EPS + 4 * rows * 2.0 ** -52))
    within(table, table_of(rows, rot, **scaling).double(), bound + gain * EPS, "table")


def turned(x, row, rot, layout, inverse=False):
    """x [..., d] in 64 bits by table rows [..., rot]: pairs as complex numbers."""
    y = x.double().clone()
    phase = torch.complex(row[..., :rot // 2].double(), row[..., rot // 2:].double())
    phase = phase.conj() if inverse else phase
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == attnw.ATTNW_HALVES else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(y[..., a], y[..., b]) * phase
    y[..., a], y[..., b] = z.real, z.imag
    return y


def bound_of(x, dtype):
    """Two products and a sum of numbers up to the largest of the pair, twice that at most; bf16 rounds once more (8 bits: by up to 2^-8 of it)."""
    return 2.0 * x.double().abs().amax(-1, keepdim=True).expand_as(x) * (3 * EPS + (2.0 ** -8 if dtype == "bf16" else 0.0)) + 1e-40


SHAPES = [(1, 1, 64, 64), (37, 3, 128, 128), (300, 2, 128, 64), (5, 16, 80, 20), (33, 1, 16, 2), (9, 4, 256, 256), (1000, 1, 64, 6), (3, 2, 72, 72), (70, 40, 48, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS])
@pytest.mark.parametrize("tokens,heads,d,rot", SHAPES)
def test_rotary(dtype, layout, tokens, heads, d, rot):
    g = torch.Generator().manual_seed(tokens + d)
    rows, t = 500, TORCH_DT[dtype]
    table = table_of(rows, rot)
    positions = torch.randint(0, rows, (tokens,), generator=g, dtype=torch.int32)
    pad = 24 if tokens % 2 else 3                 # (rows on and off the 16-byte boundaries)
    x = torch.randn((tokens, heads * d + pad), generator=g).to(t)
    dev, table_dev, pos_dev = x.cuda(), table.cuda(), positions.cuda()
    for inverse in (0, 1):
        y = torch.full((tokens, heads * d + 8), 7.0, dtype=t, device="cuda")
        attnw.attnw_rotary(dev, y, table_dev, pos_dev, tokens, heads, d, rot, rows, heads * d + pad, heads * d + 8, layout, inverse, DT[dtype])
        torch.cuda.synchronize()
        heads_of = x[:, :heads * d].view(tokens, heads, d)
        want = turned(heads_of, table[positions.long()][:, None].expand(tokens, heads, rot), rot, layout, bool(inverse))
        got = y[:, :heads * d].view(tokens, heads, d)
        within(got, want, bound_of(heads_of, dtype), "Y")
        assert torch.equal(got[..., rot:].cpu(), heads_of[..., rot:]) and bool((y[:, heads * d:] == 7).all())
        z = dev.clone()                           # in place
        attnw.attnw_rotary(z, z, table_dev, pos_dev, tokens, heads, d, rot, rows, heads * d + pad, heads * d + pad, layout, inverse, DT[dtype])
        torch.cuda.synchronize()
        assert torch.equal(z[:, :heads * d].cpu(), y[:, :heads * d].cpu()) and torch.equal(z[:, heads * d:].cpu(), x[:, heads * d:])


@pytest.mark.parametrize("layout", [attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS])
def test_gradient_against_differences(layout):
    """The map is linear: <u, f(x + h) - f(x)> is <f^T(u), h> but for rounding, with a gain in the table too."""
    g = torch.Generator().manual_seed(1)
    T, H, d, rot, rows = 11, 2, 64, 48, 300
    table = table_of(rows, rot, gain=1.25).cuda()
    positions = torch.randint(0, rows, (T,), generator=g, dtype=torch.int32).cuda()

    def f(x, inverse):
        y = torch.empty_like(x)
        attnw.attnw_rotary(x, y, table, positions, T, H, d, rot, rows, H * d, H * d, layout, inverse, attnw.ATTNW_F32)
        torch.cuda.synchronize()
        return y.double()
    x, u = (torch.randn((T, H * d), generator=g).cuda() for _ in range(2))
    for i in (0, 5, 23, 24, 47, 48, 63, 70):
        h = torch.zeros_like(x)
        h[:, i] = 0.5
        change = (f(x + h, 0) - f(x, 0)) * u.double()
        by_gradient = (f(u, 1) * h.double()).sum(1)
        # fp32 outputs of the size of a few: a rounding each
        assert float((change.sum(1) - by_gradient).abs().max()) <= 2 * H * d * 8 * EPS


def test_positions_that_the_table_does_not_have():
    table = table_of(10, 32).cuda()
    x = torch.randn((4, 64)).cuda()
    y = torch.empty_like(x)
    attnw.attnw_rotary(x, y, table, torch.tensor([3, 10, -1, 9], dtype=torch.int32).cuda(), 4, 1, 64, 32, 10, 64, 64, 0, 0, attnw.ATTNW_F32)
    torch.cuda.synchronize()
    assert torch.isnan(y[1:3, :32]).all() and torch.equal(y[:, 32:], x[:, 32:]) and torch.isfinite(y[[0, 3]]).all()


APPENDS = [
    ("one token each", [(1, 1), (1, 100), (1, 33)], 8, 2, 128, 16, 128),
    ("a ragged batch with empty ones", [(0, 5), (40, 40), (0, 0), (3, 70), (1, 129), (0, 9)], 4, 4, 64, 20, 32),
    ("columns that no vector holds", [(5, 9), (2, 2)], 3, 1, 48, 7, 22),
    ("nothing turns", [(7, 30)], 2, 2, 16, 1, 0),
    ("many sequences", [(i % 2, i % 5 + 1) for i in range(140)], 2, 1, 32, 16, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS])
@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page,rot", APPENDS, ids=[a[0] for a in APPENDS])
def test_append(dtype, layout, name, sequences, heads, kv_heads, d, page, rot):
    p = Problem(dtype, sequences, heads, kv_heads, d, page, garbage=False).on_gpu()
    g = torch.Generator().manual_seed(2)
    rows, T, t = 400, p.T, TORCH_DT[dtype]
    wide = (heads + 2 * kv_heads) * d
    x = torch.randn((T, wide), generator=g).to(t)
    q, k, v = (y.reshape(T, -1, d) for y in x.split([heads * d, kv_heads * d, kv_heads * d], 1))
    slot = torch.cat([torch.arange(m - n, m) for n, m in sequences])
    table = table_of(rows, rot) if rot else None
    for positions in (None, (slot + 13).to(torch.int32)):
        K, V = p.dev["K"].clone(), p.dev["V"].clone()
        cache = attnw.AttnwCache(K, V, p.dev["table"], p.dev["lengths"], p.batch, p.pages, p.max_pages, page, kv_heads, d, DT[dtype])
        R = torch.full((T, heads, d), 7.0, dtype=t, device="cuda")
        dev = x.cuda()
        pos_dev, table_dev = None if positions is None else positions.cuda(), None if table is None else table.cuda()
        attnw.attnw_cache_append(cache, dev, dev[:, heads * d:], dev[:, (heads + kv_heads) * d:], R, table_dev, pos_dev, p.dev["starts"], T, heads, rot,
                                 rows if rot else 0, wide, wide, layout)
        torch.cuda.synchronize()
        want_K, want_V = p.K.double().clone(), p.V.double().clone()
        K_off = torch.zeros_like(want_K)
        if rot:
            row = table[(slot if positions is None else positions.long())][:, None]
            want_q, want_k = (turned(y, row.expand(T, y.shape[1], rot), rot, layout) for y in (q, k))
            within(R, want_q, bound_of(q, dtype), "R")
        else:
            want_k = k.double()
            assert torch.equal(R.cpu(), q)
        i = 0
        for b, (n, m) in enumerate(sequences):
            for j in range(m - n, m):
                at = (p.table[b, j // page].long(), slice(None), j % page)
                want_K[at], want_V[at] = want_k[i], v[i].double()
                K_off[at] = bound_of(k[i], dtype) if rot else 0.0
                i += 1
        within(K, want_K, K_off, "K")
        assert torch.equal(V.cpu().double(), want_V)
        if positions is None:                     # keys and values alone
            K2, V2 = p.dev["K"].clone(), p.dev["V"].clone()
            cache = attnw.AttnwCache(K2, V2, p.dev["table"], p.dev["lengths"], p.batch, p.pages, p.max_pages, page, kv_heads, d, DT[dtype])
            attnw.attnw_cache_append(cache, None, dev[:, heads * d:], dev[:, (heads + kv_heads) * d:], None, table_dev, None, p.dev["starts"], T, 0, rot,
                                     rows if rot else 0, 0, wide, layout)
            torch.cuda.synchronize()
            assert torch.equal(K2, K) and torch.equal(V2, V)


def test_append_of_what_has_no_place():
    """Page ids out of range and tokens before the first slot are not cached; the others are."""
    p = Problem("bf16", [(3, 20), (2, 4)], 2, 1, 32, 16, garbage=False)
    p.table[0, 1] = 1 << 20
    p.lengths[1] = 1
    p.on_gpu()
    x = torch.randn((5, 4 * 32)).to(torch.bfloat16).cuda()
    R = torch.zeros((5, 2, 32), dtype=torch.bfloat16, device="cuda")
    before = p.dev["K"].clone()
    attnw.attnw_cache_append(p.cache, x, x[:, 64:], x[:, 96:], R, None, None, p.dev["starts"], 5, 2, 0, 0, 128, 128, 0)
    torch.cuda.synchronize()
    before[int(p.table[1, 0]), 0, 0] = x[4, 64:96]   # the second sequence's one slot
    assert torch.equal(p.dev["K"], before) and torch.equal(R.view(5, 64), x[:, :64])


def test_a_table_of_2_to_the_31_rows():
    """More rows than 31 bits count: positions of any size find theirs."""
    rows, heads, d = (1 << 31) + 5, 2, 16
    table = torch.empty((rows, 2), device="cuda")              # (16 GiB, of which a few rows are looked at)
    at = torch.tensor([0, 1, 12345, (1 << 30) + 7, (1 << 31) - 1], dtype=torch.int64, device="cuda")
    angle = torch.tensor([0.0, 0.5, 1.0, 2.0, 3.0], dtype=torch.float64)
    table[at] = torch.stack([angle.cos(), angle.sin()], 1).float().cuda()
    positions = at.to(torch.int32)
    x = torch.randn((5, heads, d), device="cuda")
    y = torch.empty_like(x)
    attnw.attnw_rotary(x, y, table, positions, 5, heads, d, 2, rows, heads * d, heads * d, attnw.ATTNW_HALVES, 0, attnw.ATTNW_F32)
    X = x.double().cpu()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    want = X.clone()
    want[..., 0], want[..., 1] = X[..., 0] * c - X[..., 1] * s, X[..., 1] * c + X[..., 0] * s
    # (cos and sin to half a unit in the last place, two products and a sum)
    bound = 4 * 2.0 ** -24 * (X[..., :2].abs().sum(-1, keepdim=True) + X.abs())
    within(y, want, bound, "y")
    starts = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    K, V = (torch.zeros((1, heads, 16, d), device="cuda") for _ in range(2))
    pages, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")
    cache = attnw.AttnwCache(K, V, pages, lengths, 1, 1, 1, 16, heads, d, attnw.ATTNW_F32)
    R = torch.empty_like(x)
    attnw.attnw_cache_append(cache, x, x, x, R, table, positions, starts, 5, heads, 2, rows, heads * d, heads * d, attnw.ATTNW_HALVES)
    within(R, want, bound, "R")
    within(K[0, :, :5].transpose(0, 1), want, bound, "K")
