"""Attention over a paged cache and the slots' sums where values or keys are infinite or no numbers: what a row sees has the part that IEEE arithmetic gives
it, wherever it lies in a tile; what it does not see has none."""
import math

import pytest
import torch

from gpu_util import require_gpu
from paged_util import Problem, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(params=[("bf16", "rows"), ("bf16", "tiles"), ("f32", "rows"), ("f32", "tiles")], ids=lambda p: "-".join(p))
def dtype(request, monkeypatch):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", request.param[1])
    return request.param[0]


VALUES = [(99, 0, 4, math.inf), (80, 2, 6, -math.inf), (62, 8, 10, math.nan), (62, 5, 6, math.inf), (71, 9, 12, math.inf), (30, 12, 14, -math.inf),
          (99, 13, 16, -math.inf)]


def expected(p, want, values):
    """The output with values that are not finite: [tokens][heads][d], 0 where only finite ones are seen, else the infinity or NaN."""
    extra = torch.zeros_like(want)
    seen = p.seen(0)
    for slot, c0, c1, kind in values:
        at = torch.zeros(want.shape[2], dtype=torch.float64)
        at[c0:c1] = kind
        extra += torch.where(seen[:, slot, None, None], at, 0.0)
    return extra


def compare(O, want, off, extra, what):
    O = O.double().cpu()
    finite = extra == 0
    assert bool(finite.any()) and not bool(finite.all())
    within(torch.where(finite, O, 0.0), torch.where(finite, want, 0.0), torch.where(finite, off, 0.0), what)
    same = (O == extra) | (torch.isnan(O) & torch.isnan(extra)) | finite
    assert bool(same.all()), f"{what}: {int((~same).sum())} values are neither the infinity nor the NaN that the definition has"


@pytest.mark.parametrize("rule", [dict(), dict(window=30), dict(window=12, prefix=[35]), dict(cap=8.0, slopes=True)], ids=["all", "window", "prefix", "cap"])
@pytest.mark.parametrize("d,page", [(64, 16), (80, 20)])
def test_infinite_values(dtype, d, page, rule):
    p = Problem(dtype, [(40, 100)], 4, 2, d, page, **rule)
    want, want_lse, off, lse_off = p.attention()
    for slot, c0, c1, kind in VALUES:
        p.V[int(p.table[0, slot // page]), :, slot % page, c0:c1] = kind
    O, lse = p.on_gpu().run_attention()
    # (columns that two of them meet in: the sum of both)
    merged = {}
    for slot, c0, c1, kind in VALUES:
        for c in range(c0, c1):
            merged[slot, c] = kind
    extra = expected(p, want, [(slot, c, c + 1, kind) for (slot, c), kind in merged.items()])
    # (the plain definition had the values that were there before; those slots' columns are judged by `extra` alone where seen)
    seen = p.seen(0)
    for (slot, c) in merged:
        assert bool((extra[seen[:, slot], :, c] != 0).all())
    compare(O, want, off, extra, "O")
    within(lse.cpu(), want_lse, lse_off, "lse")


class Some(Problem):
    """Scores of -infinity are exact."""

    def scores(self, b, h):
        x, off = super().scores(b, h)
        return x, torch.where(torch.isinf(x), 0.0, off)


def test_a_value_with_a_weight_of_nothing(dtype):
    """A slot that a row sees with a score of -infinity has a weight of 0: finite values there add nothing, NaN and infinities are NaN."""
    p = Some(dtype, [(40, 100)], 4, 2, 64, 16)
    p.Q[:, 0::64] = p.Q[:, 0::64].abs() + 0.25
    for slot, kind in ((70, math.nan), (85, math.inf)):
        page = int(p.table[0, slot // 16])
        p.K[page, :, slot % 16] = 0
        p.K[page, :, slot % 16, 0] = -math.inf
        p.V[page, :, slot % 16, 7] = kind
    O, lse = p.on_gpu().run_attention()
    want, want_lse, off, lse_off = p.attention()
    within(lse.cpu(), want_lse, lse_off, "lse")
    rows = torch.arange(60, 100)
    assert bool(torch.isnan(O.cpu()[rows >= 70][:, :, 7]).all()), "0 times NaN, 0 times infinity"
    keep = torch.ones(64, dtype=torch.bool)
    keep[7] = False
    within(O.cpu()[:, :, keep], want[:, :, keep], off[:, :, keep], "O")
    within(O.cpu()[rows < 70], want[rows < 70], off[rows < 70], "O")


def with_infinite_keys(p, slots=(70, 85, 3)):
    """Keys of some slots are -infinity in their first column, where all queries are positive: scores of -infinity, weights of 0."""
    for first in range(0, p.Q.shape[1], p.d):
        p.Q[:, first] = p.Q[:, first].abs() + 0.25
    for slot in slots:
        p.K[int(p.table[0, slot // p.page]), :, slot % p.page, 0] = -math.inf
    return p


WIDTHS = {"bf16": (16, 48, 64, 80, 112, 144, 176, 208, 240), "f32": (4, 12, 20, 36, 64, 68, 84, 100, 132, 196, 252)}


def test_infinite_keys(dtype):
    """Whatever the head size, also where a row leaves part of its place on chip empty."""
    for d in WIDTHS[dtype]:
        p = with_infinite_keys(Some(dtype, [(40, 100)], 4, 2, d, 16, seed=d))
        O, lse = p.on_gpu().run_attention()
        want, want_lse, off, lse_off = p.attention()
        within(lse.cpu(), want_lse, lse_off, f"lse, d = {d}")
        within(O.cpu(), want, off, f"O, d = {d}")


def test_infinite_keys_in_long_runs(monkeypatch):
    """(Tiles that all rows see whole: test_gpu_paged_segments.)"""
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", "tiles")
    for d in (16, 48, 80, 112, 144):
        p = with_infinite_keys(Some("bf16", [(300, 4000)], 192, 96, d, 32, seed=d, garbage=False), (70, 1500, 3901))
        O, lse = p.on_gpu().run_attention()
        want, want_lse, off, lse_off = p.attention()
        within(lse.cpu(), want_lse, lse_off, f"lse, d = {d}")
        within(O.cpu(), want, off, f"O, d = {d}")


@pytest.mark.parametrize("new", [1, 300])
@pytest.mark.parametrize("of", ["bf16", "f32"])
def test_infinite_keys_of_sums(of, new):
    """(300 tokens: rows in turns, else held.)"""
    for d in WIDTHS[of]:
        p = with_infinite_keys(Some(of, [(new, 400)], 4, 2, d, 16, seed=d)).on_gpu()
        _, lse, _, _ = p.attention()
        want, bound = p.collected(lse.float(), None)
        within(p.run_sums(lse.float().cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, f"sums, d = {d}")


def test_small_queries(dtype):
    """Queries of all sizes down to the least normal number: what is shared out between two places on chip adds up."""
    for d in WIDTHS[dtype]:
        p = Problem(dtype, [(40, 100)], 4, 2, d, 16, seed=d)
        g = torch.Generator().manual_seed(d)
        p.Q = p.Q.sign() * torch.exp2(torch.randint(-126, -108, p.Q.shape, generator=g).float()).to(p.Q.dtype) * (1.0 + 0.5 * torch.rand(p.Q.shape, generator=g)).to(p.Q.dtype)
        p.K = torch.where(torch.isfinite(p.K), p.K * 2.0 ** 110, p.K)
        p.scale = 2.0 ** -4
        O, lse = p.on_gpu().run_attention()
        want, want_lse, off, lse_off = p.attention()
        assert float((want_lse[:, 0] - want_lse[:, 1]).abs().max()) > 1e-4
        within(lse.cpu(), want_lse, lse_off, f"lse, d = {d}")
        within(O.cpu(), want, off, f"O, d = {d}")
        want, bound = p.collected(lse.cpu(), None)
        within(p.run_sums(lse, None, torch.zeros(want.shape, device="cuda")), want, bound, f"sums, d = {d}")


# ---- caps ---------------------------------------------------------------------------------------------------------------------------------

class Capped(Problem):
    """The same, with what fp32 may be off by in terms of the score, not of the cap."""

    def scores(self, b, h):
        cap, self.cap = self.cap, 0.0
        x, off = super().scores(b, h)
        self.cap = cap
        seen = self.seen(b)
        y = cap * torch.tanh(torch.where(seen, x, 0.0) / cap)
        # 1 - 2 / (2^z + 1) is off by 2^-22 (a unit in the last place each of exponential and reciprocal, half of one of the sum and of z): 2^-20 of tanh from a quarter
        # on, and with the roundings of what it is multiplied by 2^-19; below a quarter, and by tanhf, less.  Caps up to 128 may be made so everywhere.
        own = 2.0 ** -19 * y.abs() if cap > 128.0 else torch.full_like(y, cap * 2.0 ** -22)
        return y.masked_fill(~seen, -math.inf), off + own + 8 * 2.0 ** -24 * y.abs()


@pytest.mark.parametrize("cap", [1e-40, 1e-3, 30.0, 128.0, 129.0, 1000.0, 1e5, 1e30, 3e38])
@pytest.mark.parametrize("sharp", [1.0, 40.0])
def test_caps(dtype, cap, sharp):
    """However large the cap: scores are as exact as their own size lets them be."""
    p = Capped(dtype, [(40, 300)], 4, 2, 64, 16, cap=cap, sharp=sharp)
    O, lse = p.on_gpu().run_attention()
    want, want_lse, off, lse_off = p.attention()
    within(lse.cpu(), want_lse, lse_off, "lse")
    within(O.cpu(), want, off, "O")
    for new in (40, 150):                         # (held rows, rows in turn)
        p = Capped(dtype, [(new, 300)], 4, 2, 64, 16, cap=cap, sharp=sharp).on_gpu()
        _, lse, _, _ = p.attention()
        want, bound = p.collected(lse.float(), None)
        within(p.run_sums(lse.float().cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, f"sums of {new}")


@pytest.mark.parametrize("cap", [128.0, 200.0])
def test_caps_in_long_runs(monkeypatch, cap):
    """(Workgroups with two places of 128 keys and more: the order in which tiles that all rows see go up to a cap of 128.)"""
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", "tiles")
    p = Capped("bf16", [(300, 2500)], 24, 24, 128, 32, cap=cap, sharp=20.0)
    O, lse = p.on_gpu().run_attention()
    want, want_lse, off, lse_off = p.attention()
    within(lse.cpu(), want_lse, lse_off, "lse")
    within(O.cpu(), want, off, "O")


@pytest.mark.parametrize("of", ["bf16", "f32"])
@pytest.mark.parametrize("new", [3, 20, 300])
def test_sums_of_rows_that_do_not_count(of, new):
    """Rows whose lse is -infinity add nothing, whatever their queries are: padding may hold anything."""
    for d in (64, 80):
        p = Problem(of, [(new, 400)], 4, 2, d, 16, seed=d)
        _, lse, _, _ = p.attention()
        lse = lse.float()
        for t, h, kind in ((0, 0, math.nan), (new - 1, 3, math.inf), (new // 2, 1, -math.inf), (new - 1, 2, math.nan)):
            p.Q[t, h * d:(h + 1) * d] = kind
            lse[t, h] = -math.inf
        clean = Problem(of, [(new, 400)], 4, 2, d, 16, seed=d)
        want, bound = clean.collected(lse, None)
        p.on_gpu()
        within(p.run_sums(lse.cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, f"sums, d = {d}")
