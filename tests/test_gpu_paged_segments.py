"""Paged attention and sums where one workgroup has much to do: tiles in long runs, lists of keys longer than what is kept on chip, several blocks of
keys of one workgroup, the chunk kernel in fp32 and with pages of every kind.  Against the definitions in 64 bits (paged_util), evaluated on the device."""
import math

import pytest
import torch

import paper_2407_13885_amd as attnw
from gpu_util import TORCH_DT, kernels, require_gpu
from paged_util import Problem, within
from test_gpu_paged import RULES, SHAPES, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(params=["rows", "tiles"])
def kernel(request, monkeypatch):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", request.param)
    return request.param


@pytest.fixture
def tiles(monkeypatch):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", "tiles")


class OnDevice(Problem):
    """The same problem, its definition in 64 bits evaluated on the device."""

    def __init__(self, *args, **more):
        super().__init__(*args, **more)
        for k, v in list(vars(self).items()):
            if isinstance(v, torch.Tensor):
                setattr(self, k, v.cuda())

    def attention(self):
        with torch.device("cuda"):
            return [x.cpu() for x in super().attention()]

    def collected(self, lse, before):
        with torch.device("cuda"):
            return [x.cpu() for x in super().collected(lse, before)]


def compute_units():
    return torch.cuda.get_device_properties(0).multi_processor_count


def places(p, rows, unit):
    """Places of the work list of attention without a window: blocks of `rows` rows, one place for each `unit` keys of a sequence."""
    return sum(-(-n * p.group // rows) * max(1, -(-m // unit)) * p.kv_heads for n, m in p.sequences)


def least_keys(p, rows, unit):
    """Keys of a workgroup's stretch at least, whatever the kernel: two workgroups a compute unit at most."""
    return places(p, rows, unit) // (2 * compute_units()) * unit


# ---- chunks in long runs ------------------------------------------------------------------------------------------------------------------
# bf16 blocks of 128 rows; a run without masks takes six tiles of 32 keys at least: here 20 to 40 of them, ends of any parity, last blocks of few rows

LONG = [(1023, 5300), (70, 70), (37, 6150)]


@pytest.mark.parametrize("d,page", [(16, 16), (32, 20), (64, 16), (64, 64), (80, 64), (96, 32), (112, 16), (128, 16), (128, 48), (128, 20), (144, 32), (160, 64)])
def test_long_runs(tiles, d, page):
    p = OnDevice("bf16", LONG, 48, 12, d, page, seed=d + page)
    assert least_keys(p, 128, 128) >= 5 * 128
    check_attention(p)


@pytest.mark.parametrize("d", [64, 80, 128, 160])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_rules_of_long_runs(tiles, d, name, more):
    """(A window of 50 or less leaves no run; prefixes of hundreds do.)"""
    more = dict(more)
    if "prefix" in more:
        more["prefix"] = [2500, 33, 4100]
    if more.get("window", 0) == 70:
        more["window"] = 2900
    p = OnDevice("bf16", LONG, 48, 12, d, 64 if d % 64 else 16, seed=3, **more)
    assert least_keys(p, 128, 128) >= 5 * 128
    check_attention(p)


def test_waves_without_rows_in_long_runs(tiles):
    """Blocks of 8, of 40 and of 100 rows: some waves of a workgroup only move tiles."""
    for new, group in ((8, 1), (8, 5), (25, 4)):
        p = OnDevice("bf16", [(new, 9001), (1, 8000)], 32 * group, 32, 64, 32, seed=group)
        assert least_keys(p, 128, 128) >= 5 * 128
        check_attention(p)


@pytest.mark.parametrize("window", [33, 1000, 3001])
def test_windows_of_long_runs(tiles, window):
    check_attention(OnDevice("bf16", LONG, 48, 12, 128, 16, window=window, seed=window))


def test_rows_of_rising_scores(tiles):
    """Keys that match the better the later they come: the exponent moves all along the run."""
    p = OnDevice("bf16", LONG, 48, 12, 64, 16, seed=1, garbage=False)
    for b, (_, m) in enumerate(p.sequences):
        j = torch.arange(m, device="cuda")
        p.K[p.table[b, j // 16].long(), :, j % 16, 0] = (8.0 * j / m).to(torch.bfloat16)[:, None]
    p.Q[:, 0::64] = 40.0                          # (rises by 40 in all: 58 binades, the lazy bound is 6)
    check_attention(p)


# ---- chunks in fp32 -----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page", SHAPES, ids=[s[0] for s in SHAPES])
def test_shapes_of_chunks_in_f32(tiles, name, sequences, heads, kv_heads, d, page):
    check_attention(Problem("f32", sequences, heads, kv_heads, d, page, seed=len(name)))


@pytest.mark.parametrize("d", [4, 12, 16, 20, 32, 36, 48, 52, 64, 68, 80, 84, 96, 100, 128, 132, 192, 196, 252, 256])
def test_head_sizes_of_chunks_in_f32(tiles, d):
    check_attention(Problem("f32", [(1, 190), (50, 775)], 4, 2, d, 16 if d % 64 else 24, seed=d))


@pytest.mark.parametrize("d", [64, 80])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_rules_of_chunks_in_f32(tiles, d, name, more):
    check_attention(Problem("f32", [(1, 410), (40, 333), (150, 1020)], 8, 4, d, 32, seed=3, **more))


def test_sizes_lead_to_chunks_in_f32():
    p = OnDevice("f32", [(197, 1222), (60, 400), (150, 1100)], 16, 8, 80, 20, seed=2)
    check_attention(p)
    work = torch.empty(attnw.attnw_paged_workspace(p.cache, p.T, 16), dtype=torch.uint8, device="cuda")
    O, d = torch.empty((p.T, 16, 80), device="cuda"), p.dev
    ran = kernels(lambda s: attnw.attnw_paged_attention(p.cache, p.rule, d["Q"], O, None, d["starts"], p.T, 16, p.q_stride, work, work.numel(), s))
    assert "paged_tiles_kernelIf" in ran[0]


@pytest.mark.parametrize("d,page", [(32, 16), (64, 20), (128, 64), (256, 16)])
def test_long_stretches_in_f32(tiles, d, page):
    p = OnDevice("f32", [(333, 3300), (70, 70), (37, 3150)], 32, 8, d, page, seed=d)
    assert least_keys(p, 64, 64) >= 5 * 64
    check_attention(p)


def test_hidden_values_of_chunks_in_f32(tiles):
    for window, prefix in ((0, None), (30, None), (12, [5])):
        p = Problem("f32", [(40, 100)], 4, 2, 64, 16, window=window, prefix=prefix)
        slots = [99, 80, 62]
        for slot, kind in zip(slots, (math.nan, math.inf, -math.inf)):
            page = int(p.table[0, slot // 16])
            p.V[page, :, slot % 16, 3:9] = kind
            p.K[page, 1, slot % 16] = math.nan
        O, lse = p.on_gpu().run_attention()
        want, want_lse, off, lse_off = p.attention()
        hidden = ~p.seen(0)[:, slots].any(1)
        within(O.cpu()[hidden], want[hidden], off[hidden], "O")
        within(lse.cpu()[hidden], want_lse[hidden], lse_off[hidden], "lse")


# ---- pages of one slot: more keys of a workgroup than places are kept on chip (1024) ----------------------------------------------------------

def test_more_places_than_are_kept_on_chip(kernel):
    # 128 kv heads and 12000 slots: blocks of 16 rows 47 places of 256 keys each, 11 of them a workgroup; of 128 rows 94 of 128
    p = OnDevice("bf16", [(3, 12000)], 256, 128, 16, 1)
    assert least_keys(p, *((16, 256) if kernel == "rows" else (128, 128))) >= 2 * 1024
    check_attention(p)


@pytest.mark.parametrize("new", [1, 300])
def test_sums_of_many_blocks_and_places(new):
    """Workgroups with several blocks of keys of several kv heads; single tokens (held rows, tiles in a ring) and chunks (rows in turn)."""
    p = OnDevice("bf16", [(new, 15000), (new, 2100)], 256, 256, 16, 1, garbage=False).on_gpu()
    keys, workgroups = (128, 4) if new == 1 else (64, 16)
    assert sum(-(-m // keys) for _, m in p.sequences) * 256 // (workgroups * compute_units()) * keys >= 1024
    _, lse, _, _ = p.attention()
    lse = lse.float()
    before = torch.rand((2, 256, p.max_pages))
    for b in (before, None):
        want, bound = p.collected(lse.cuda(), None if b is None else b.cuda())
        for in_place in ((False, True) if b is not None else (False,)):
            sums = b.clone().cuda() if in_place else torch.zeros(before.shape, device="cuda")
            p.run_sums(lse.cuda(), sums if in_place else None if b is None else b.cuda(), sums)
            for i, (_, m) in enumerate(p.sequences):
                within(sums[i, :, :m], want[i, :, :m], bound[i, :, :m], f"sums {in_place}")


@pytest.mark.parametrize("dtype,d,page,more", [("bf16", 64, 16, {}), ("bf16", 256, 20, dict(cap=9.0)), ("f32", 64, 32, dict(slopes=True)), ("f32", 132, 16, {}),
                                               ("bf16", 128, 16, dict(window=1500, prefix=[700, 0]))])
@pytest.mark.parametrize("new", [1, 130])
def test_sums_of_many_blocks(dtype, d, page, more, new):
    """(130 tokens of a group of 2: 260 rows of a sequence, beyond either type's rule for held ones.)"""
    p = OnDevice(dtype, [(new, 9000), (new, 4321)], 128, 64, d, page, seed=d, garbage=False, **more).on_gpu()
    _, lse, _, _ = p.attention()
    want, bound = p.collected(lse.float().cuda(), None)
    sums = torch.zeros(want.shape, device="cuda")
    # (at most 128 keys a block, 4 workgroups a compute unit; in turns 64 and 16)
    assert sum(-(-m // (128 if new == 1 else 64)) for _, m in p.sequences) * 64 > (4 if new == 1 else 16) * compute_units()
    within(p.run_sums(lse.float().cuda(), None, sums), want, bound, "sums")
    O, got_lse = p.run_attention()
    assert TORCH_DT[dtype] == O.dtype


# ---- which kernel -------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,tokens,heads,kv_heads,d,want", [
    ("bf16", 64, 32, 8, 256, "tiles"),            # measured at 4096 and 16384 slots, us, small blocks / large ones: 96 / 64, 334 / 108
    ("bf16", 128, 4, 1, 256, "rows"),             # 37 / 55, 98 / 94
    ("bf16", 64, 64, 16, 64, "rows"),             # 22 / 56, 63 / 70
    ("bf16", 256, 32, 8, 64, "tiles"),            # 39 / 39, 118 / 66
    ("f32", 32, 64, 16, 64, "rows"),              # 36 / 54, 112 / 126
    ("f32", 64, 16, 4, 256, "tiles"),             # 135 / 86, 478 / 244
    ("bf16", 1, 32, 8, 128, "rows"),
])
def test_the_kernel_that_sizes_lead_to(dtype, tokens, heads, kv_heads, d, want):
    p = Problem(dtype, [(tokens, 4096)], heads, kv_heads, d, 64, garbage=False).on_gpu()
    work = torch.empty(attnw.attnw_paged_workspace(p.cache, tokens, heads), dtype=torch.uint8, device="cuda")
    O, dev = torch.empty((tokens, heads, d), dtype=TORCH_DT[dtype], device="cuda"), p.dev
    ran = kernels(lambda s: attnw.attnw_paged_attention(p.cache, p.rule, dev["Q"], O, None, dev["starts"], tokens, heads, p.q_stride, work, work.numel(), s))
    assert f"paged_{want}_kernel" in ran[0]


# ---- scales, and batches of more sequences than a wave has lanes ------------------------------------------------------------------------------

class Scaled(OnDevice):
    """A scale of either sign: what fp32 may be off by goes with its size."""

    def scores(self, b, h):
        scale, self.scale = self.scale, abs(self.scale)
        off = super().scores(b, h)[1]
        self.scale = scale
        x, own = super().scores(b, h)
        return x, torch.maximum(off, own.abs())


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-30, 2.0])
def test_scales(kernel, scale, cap):
    p = Scaled("bf16", [(300, 2500), (3, 70)], 24, 24, 64, 32, seed=4, cap=cap)
    p.scale = scale
    O, lse = check_attention(p)
    before = torch.rand((2, 24, p.max_pages * 32))
    want, bound = p.collected(lse, before.cuda())
    sums = p.run_sums(lse, before.cuda(), torch.zeros(want.shape, device="cuda"))
    for b, (_, m) in enumerate(p.sequences):
        within(sums[b, :, :m], want[b, :, :m], bound[b, :, :m], "sums")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,most", [(1, 2000), (3, 500), (90, 700)])
def test_many_sequences_of_either_kernel(kernel, dtype, new, most):
    sequences = [((i * 7) % (new + 1), max((i * 7) % (new + 1), (i * 37) % most + 2)) for i in range(150)]
    p = OnDevice(dtype, sequences, 4, 2, 32, 16, seed=new)
    O, lse = check_attention(p)
    want, bound = p.collected(lse, None)
    sums = p.run_sums(lse, None, torch.zeros(want.shape, device="cuda"))
    for b, (_, m) in enumerate(p.sequences):
        within(sums[b, :, :m], want[b, :, :m], bound[b, :, :m], "sums")
