"""Attention over a paged cache, the weight that slots collect, and eviction, against their definitions in 64 bits (paged_util)."""
import math

import numpy as np
import pytest
import torch

import paper_2407_13885_amd as attnw
from gpu_util import DT, TORCH_DT, kernels, require_gpu
from paged_util import Problem, evicted, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def check_attention(p):
    O, lse = p.on_gpu().run_attention()
    want, want_lse, off, lse_off = p.attention()
    within(O[:p.T], want, off, "O")
    within(lse[:p.T], want_lse, lse_off, "lse")
    return O, lse


# sequences (new, in use), heads, kv heads, d, page
SHAPES = [
    ("one token alone", [(1, 1)], 1, 1, 64, 16),
    ("one token, odd length", [(1, 777)], 8, 2, 128, 16),
    ("one token, a long row", [(1, 5001)], 4, 1, 64, 64),
    ("tokens of several lengths, some empty", [(1, 1), (0, 40), (1, 33), (1, 640), (0, 0), (1, 129)], 8, 4, 128, 32),
    ("a chunk at the start", [(37, 37)], 4, 4, 64, 16),
    ("a chunk over others", [(65, 300), (3, 259), (128, 128)], 8, 2, 128, 20),
    ("groups that blocks cut", [(19, 90), (5, 5)], 21, 3, 32, 7),
    ("more heads than a block has rows", [(2, 70), (1, 513)], 48, 1, 64, 128),
    ("pages of one slot", [(4, 101)], 2, 1, 16, 1),
    ("more pages than are kept on chip", [(2, 2600)], 2, 1, 16, 1),
    ("a long chunk", [(300, 812)], 2, 1, 128, 48),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page", SHAPES, ids=[s[0] for s in SHAPES])
def test_attention(dtype, name, sequences, heads, kv_heads, d, page):
    check_attention(Problem(dtype, sequences, heads, kv_heads, d, page, seed=len(name)))


@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in (16, 48, 80, 96, 112, 144, 160, 176, 192, 208, 224, 256)]
                         + [("f32", d) for d in (4, 12, 20, 36, 68, 100, 132, 196, 252, 256)])
def test_head_sizes(dtype, d):
    check_attention(Problem(dtype, [(1, 190), (18, 75)], 4, 2, d, 16, seed=d))


@pytest.fixture(params=["rows", "tiles"])
def kernel(request, monkeypatch):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", request.param)
    return request.param


def test_either_kernel_of_a_shape(kernel):
    p = Problem("bf16", [(1, 300), (9, 9)], 4, 2, 64, 16).on_gpu()
    work = torch.empty(attnw.attnw_paged_workspace(p.cache, p.T, 4), dtype=torch.uint8, device="cuda")
    O, d = torch.empty((p.T, 4, 64), dtype=torch.bfloat16, device="cuda"), p.dev
    ran = kernels(lambda s: attnw.attnw_paged_attention(p.cache, p.rule, d["Q"], O, None, d["starts"], p.T, 4, p.q_stride, work, work.numel(), s))
    assert f"paged_{kernel}_kernel" in ran[0]


@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page", SHAPES, ids=[s[0] for s in SHAPES])
def test_shapes_of_either_kernel(kernel, name, sequences, heads, kv_heads, d, page):
    check_attention(Problem("bf16", sequences, heads, kv_heads, d, page, seed=len(name)))


@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 112, 128, 144, 160, 176, 192, 208, 256])
def test_head_sizes_of_either_kernel(kernel, d):
    check_attention(Problem("bf16", [(1, 190), (50, 775)], 4, 2, d, 16 if d % 64 else 24, seed=d))


RULES = [
    ("cap", dict(cap=5.0, sharp=3.0)),
    ("bias by distance", dict(slopes=True)),
    ("cap and bias", dict(cap=20.0, slopes=True)),
    ("window of one", dict(window=1)),
    ("window", dict(window=50)),
    ("prefix", dict(prefix=[0, 33, 400])),
    ("window and prefix", dict(window=20, prefix=[17, 300, 1])),
    ("everything", dict(cap=9.0, slopes=True, window=70, prefix=[90, 0, 64])),
    ("sharp rows", dict(sharp=30.0)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_rules(dtype, name, more):
    check_attention(Problem(dtype, [(1, 410), (40, 333), (150, 420)], 8, 4, 64, 32, seed=3, **more))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(dtype):
    """A sequence of more tokens than slots: those before its first slot see the prefix or nothing."""
    p = Problem(dtype, [(4, 60)], 4, 2, 64, 16, more_pages=1)
    p.lengths[0] = 2
    O, lse = p.on_gpu().run_attention()
    q = Problem(dtype, [(2, 2)], 4, 2, 64, 16)
    q.table, q.K, q.V, q.pages = p.table, p.K, p.V, p.pages
    q.Q = p.Q[2:]
    want, want_lse, off, lse_off = q.attention()
    assert bool((O[:2] == 0).all()) and bool(torch.isneginf(lse[:2]).all())
    within(O[2:], want, off, "O")
    within(lse[2:], want_lse, lse_off, "lse")
    p = Problem(dtype, [(3, 0)], 4, 2, 64, 16, more_pages=1)      # no slot at all
    O, lse = p.on_gpu().run_attention()
    assert bool((O == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("dtype,kernel_of", [("bf16", "rows"), ("bf16", "tiles"), ("f32", "")])
def test_what_is_hidden_has_no_part(dtype, kernel_of, monkeypatch):
    """Keys and values of tokens that a row does not see may hold NaN and infinity: later ones of its chunk, ones in front of its window."""
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", kernel_of)
    for window, prefix in ((0, None), (30, None), (12, [5])):
        p = Problem(dtype, [(40, 100)], 4, 2, 64, 16, window=window, prefix=prefix)
        for slot, kind in ((99, math.nan), (80, math.inf), (62, -math.inf)):
            page = int(p.table[0, slot // 16])
            p.V[page, :, slot % 16, 3:9] = kind
            p.K[page, 1, slot % 16] = math.nan
        O, lse = p.on_gpu().run_attention()
        want, want_lse, off, lse_off = p.attention()
        # (a token's own row sees these slots if it stands at or behind them: then it is not compared)
        hidden = ~p.seen(0)[:, [99, 80, 62]].any(1)
        assert 1 < int(hidden.sum()) < 40
        within(O.cpu()[hidden], want[hidden], off[hidden], "O")
        within(lse.cpu()[hidden], want_lse[hidden], lse_off[hidden], "lse")
        exposed = O.cpu()[~hidden][:, :, 3:9].float()
        assert not bool(torch.isfinite(exposed).any()), "a row that sees a NaN has one"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_strided_projection_and_another_stream(dtype):
    p = Problem(dtype, [(5, 200), (1, 64)], 6, 2, 64, 16, q_pad=4 * 64).on_gpu()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O, lse = p.run_attention(side)
    want, want_lse, off, lse_off = p.attention()
    within(O, want, off, "O")
    within(lse, want_lse, lse_off, "lse")


def test_the_same_bits_every_time():
    p = Problem("bf16", [(1, 3000), (1, 17), (60, 900)], 16, 4, 128, 16).on_gpu()
    first = p.run_attention()
    for _ in range(3):
        again = p.run_attention()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_contents_out_of_range_stay_in_range():
    """Lengths, starts and page ids that no host can check: nothing outside the arrays is touched, other sequences are as they were."""
    p = Problem("bf16", [(1, 100), (2, 90), (1, 64)], 4, 2, 64, 16, garbage=False)
    want, want_lse, off, lse_off = p.attention()
    p.table[1, 0], p.table[1, 1] = -5, 1 << 30
    p.lengths[1] = 1 << 30
    O, lse = p.on_gpu().run_attention()
    for rows in (slice(0, 1), slice(3, 4)):
        within(O[rows], want[rows], off[rows], "O")
    p.lengths[1] = -7
    O, lse = p.on_gpu().run_attention()
    within(O[3:], want[3:], off[3:], "O")
    assert bool((O[1:3] == 0).all())


@pytest.mark.parametrize("batch", [3, 100])
def test_starts_in_no_order(batch):
    """Sequences that claim each other's tokens, and tokens that there are not: any of the rows, but nothing outside the arrays."""
    p = Problem("bf16", [(2, 50 + b % 7) for b in range(batch)], 4, 2, 64, 16, garbage=False)
    p.starts = torch.tensor([(-3, 0, p.T, (1 << 31) - 1, 2, -(1 << 31), 7)[b % 7] for b in range(batch + 1)], dtype=torch.int32)
    O, lse = p.on_gpu().run_attention()
    sums = torch.zeros((batch, 2, p.max_pages * 16), device="cuda")
    p.run_sums(torch.nan_to_num(lse, neginf=0.0), None, sums)
    assert O.shape[0] == p.T and bool(torch.isfinite(O).all()) and bool(torch.isfinite(sums).all())


def test_offsets_beyond_32_bits():
    """The last pages of a cache of more than 4 GiB of keys."""
    p = Problem("bf16", [(1, 70)], 2, 1, 256, 16)
    pages = (1 << 32) // (16 * 256 * 2) + 40
    K = torch.empty((pages, 1, 16, 256), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    where = torch.tensor([pages - 1 - 3 * i for i in range(p.max_pages)])
    K[where.cuda()] = p.K[p.table[0].long()].cuda()
    V[where.cuda()] = p.V[p.table[0].long()].cuda()
    want, want_lse, off, lse_off = p.attention()
    p.table = where.to(torch.int32).view(1, -1)
    p.on_gpu()
    p.cache = attnw.AttnwCache(K, V, p.dev["table"], p.dev["lengths"], 1, pages, p.max_pages, 16, 1, 256, attnw.ATTNW_BF16)
    O, lse = p.run_attention()
    within(O, want, off, "O")
    sums = torch.zeros((1, 1, p.max_pages * 16), device="cuda")
    want_sums, bound = Problem("bf16", [(1, 70)], 2, 1, 256, 16).collected(lse.cpu(), None)
    within(p.run_sums(lse, None, sums), want_sums, bound, "sums")


def test_many_sequences():
    """More sequences than lanes, most of them short."""
    sequences = [((i * 7) % 3, (i * 37) % 90 + 2) for i in range(150)]
    p = Problem("bf16", sequences, 4, 2, 32, 16)
    O, lse = check_attention(p)
    want, bound = p.collected(lse.cpu(), None)
    within(p.run_sums(lse, None, torch.zeros(want.shape, device="cuda")), want, bound, "sums")


def test_recorded_and_replayed():
    """A recorded step follows lengths that change between the replays."""
    p = Problem("bf16", [(1, 600), (1, 350)], 8, 2, 128, 16, more_pages=2, garbage=False).on_gpu()
    d = p.dev
    O, lse = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8), device="cuda")
    sums = torch.zeros((2, 2, p.max_pages * 16), device="cuda")
    size = attnw.attnw_paged_workspace(p.cache, 2, 8)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        attnw.attnw_paged_attention(p.cache, p.rule, d["Q"], O, lse, d["starts"], 2, 8, p.q_stride, work, size, stream)
        attnw.attnw_paged_sums(p.cache, p.rule, d["Q"], lse, None, sums, d["starts"], 2, 8, p.q_stride, stream)
    for lengths in ((600, 350), (601, 5), (33, 364), (610, 64)):
        p.sequences = [(1, m) for m in lengths]
        p.lengths = torch.tensor(lengths, dtype=torch.int32)
        d["lengths"].copy_(p.lengths)
        sums.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse, off, lse_off = p.attention()
        within(O, want, off, "O")
        within(lse, want_lse, lse_off, "lse")
        want, bound = p.collected(lse.cpu(), None)
        within(sums, want, bound, "sums")


@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_rules_of_either_kernel(kernel, name, more):
    check_attention(Problem("bf16", [(1, 410), (40, 333), (150, 1020)], 8, 4, 64, 32, seed=3, **more))


# ---- the weight that slots collect --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page", SHAPES, ids=[s[0] for s in SHAPES])
def test_sums(dtype, name, sequences, heads, kv_heads, d, page):
    p = Problem(dtype, sequences, heads, kv_heads, d, page, seed=len(name)).on_gpu()
    _, lse, _, _ = p.attention()
    lse = lse.float()
    before = torch.rand((p.batch, p.kv_heads, p.max_pages * p.page))
    want, bound = p.collected(lse, before)
    sums = before.clone().cuda()
    p.run_sums(lse.cuda(), sums, sums)            # in place
    for b, (n, m) in enumerate(sequences):
        within(sums[b, :, :m], want[b, :, :m], bound[b, :, :m], "sums")
        assert torch.equal(sums[b, :, m:].cpu(), before[b, :, m:]), "slots that are not in use"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_sums_of_rules(dtype, name, more):
    p = Problem(dtype, [(1, 410), (40, 333), (150, 420)], 8, 4, 64, 32, seed=3, **more).on_gpu()
    _, lse, _, _ = p.attention()
    want, bound = p.collected(lse.float(), None)
    sums = torch.zeros(want.shape, device="cuda")
    within(p.run_sums(lse.float().cuda(), None, sums), want, bound, "sums")


@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in (16, 80, 144, 256)] + [("f32", d) for d in (4, 36, 100, 252)])
def test_sums_of_head_sizes(dtype, d):
    p = Problem(dtype, [(1, 190), (18, 75)], 4, 2, d, 16, seed=d).on_gpu()
    _, lse, _, _ = p.attention()
    want, bound = p.collected(lse.float(), None)
    within(p.run_sums(lse.float().cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, "sums")


def test_sums_of_rows_that_see_nothing():
    p = Problem("bf16", [(4, 60)], 4, 2, 64, 16, more_pages=1)
    p.lengths[0] = 2
    p.on_gpu()
    lse = torch.full((4, 4), -math.inf, device="cuda")
    sums = p.run_sums(lse, None, torch.full((1, 2, p.max_pages * 16), 5.0, device="cuda"))
    assert bool((sums[:, :, :2] == 0).all()) and bool((sums[:, :, 2:] == 5).all())


# (long enough that waves take rows in turns, in either type)
LONG = [
    ("one chunk", [(600, 777)], 2, 2, 64, 16),
    ("beside others and none", [(700, 900), (0, 40), (3, 65), (0, 0), (513, 513)], 8, 4, 128, 20),
    ("groups that blocks cut", [(95, 190), (61, 61)], 21, 3, 32, 7),
    ("pages of one slot", [(300, 1101)], 2, 1, 16, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,sequences,heads,kv_heads,d,page", LONG, ids=[s[0] for s in LONG])
def test_sums_of_long_chunks(dtype, name, sequences, heads, kv_heads, d, page):
    test_sums(dtype, name, sequences, heads, kv_heads, d, page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_sums_of_rules_and_long_chunks(dtype, name, more):
    p = Problem(dtype, [(1, 410), (40, 333), (400, 620)], 8, 4, 64, 32, seed=3, **more).on_gpu()
    _, lse, _, _ = p.attention()
    want, bound = p.collected(lse.float(), None)
    within(p.run_sums(lse.float().cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, "sums")


@pytest.mark.parametrize("dtype,d", [("bf16", d) for d in (16, 80, 144, 256)] + [("f32", d) for d in (4, 36, 100, 252)])
def test_sums_of_head_sizes_and_long_chunks(dtype, d):
    p = Problem(dtype, [(1, 190), (290, 375)], 4, 2, d, 16, seed=d).on_gpu()
    _, lse, _, _ = p.attention()
    want, bound = p.collected(lse.float(), None)
    within(p.run_sums(lse.float().cuda(), None, torch.zeros(want.shape, device="cuda")), want, bound, "sums")


def test_sums_of_long_chunks_that_see_nothing():
    p = Problem("bf16", [(400, 460)], 4, 2, 64, 16, more_pages=1)
    p.lengths[0] = 2
    p.on_gpu()
    lse = torch.full((400, 4), -math.inf, device="cuda")
    sums = p.run_sums(lse, None, torch.full((1, 2, p.max_pages * 16), 5.0, device="cuda"))
    assert bool((sums[:, :, :2] == 0).all()) and bool((sums[:, :, 2:] == 5).all())


# ---- eviction -----------------------------------------------------------------------------------------------------------------------------

def check_eviction(dtype, lengths, kv_heads, d, page, keep, recent, sums, into_page=None, more_pages=0):
    p = Problem(dtype, [(0, m) for m in lengths], kv_heads, kv_heads, d, page, garbage=False, more_pages=more_pages).on_gpu()
    into_page = into_page or page
    slots = p.max_pages * page
    x = np.zeros((p.batch, kv_heads, slots), np.float32)
    for b, m in enumerate(lengths):
        x[b, :, :m] = sums(b, kv_heads, m)
    most = -(-keep // into_page)
    pages = p.batch * most + 2
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(5))[:p.batch * most].to(torch.int32).view(p.batch, most)
    t = TORCH_DT[dtype]
    K, V = (torch.full((pages, kv_heads, into_page, d), 7.0, dtype=t, device="cuda") for _ in range(2))
    into_sums = torch.full((p.batch, kv_heads, most * into_page), 7.0, device="cuda")
    kept = torch.full((p.batch, kv_heads, keep), 77, dtype=torch.int32, device="cuda")
    into_lengths = torch.full((p.batch,), 77, dtype=torch.int32, device="cuda")
    dev_table = table.cuda()
    into = attnw.AttnwCache(K, V, dev_table, into_lengths, p.batch, pages, most, into_page, kv_heads, d, DT[dtype])
    attnw.attnw_cache_evict(p.cache, into, torch.from_numpy(x).cuda(), into_sums, kept, keep, recent)
    torch.cuda.synchronize()
    want = evicted(x, lengths, keep, recent)
    assert np.array_equal(kept.cpu().numpy(), want)
    assert into_lengths.tolist() == [min(m, keep) for m in lengths]
    want_K, want_V = (torch.full((pages, kv_heads, into_page, d), 7.0, dtype=t) for _ in range(2))
    want_sums = np.full(into_sums.shape, 7.0, np.float32)
    for b, m in enumerate(lengths):
        for h in range(kv_heads):
            slot = want[b, h][want[b, h] >= 0].astype(np.int64)
            to = np.arange(len(slot))
            want_sums[b, h, :len(slot)] = x[b, h, slot]
            for src, dst in ((p.K, want_K), (p.V, want_V)):
                dst[table[b].long()[to // into_page], h, to % into_page] = src[p.table[b].long()[slot // page], h, slot % page]
    assert torch.equal(K.cpu(), want_K) and torch.equal(V.cpu(), want_V)
    assert np.array_equal(into_sums.cpu().numpy(), want_sums, equal_nan=True)


def _heavy(b, h, m):
    return np.exp(2.0 * np.random.default_rng(b + m).standard_normal((h, m))).astype(np.float32)


def _ties(b, h, m):
    return np.random.default_rng(b).integers(0, 3, (h, m)).astype(np.float32)


def _odd(b, h, m):
    x = np.random.default_rng(b).standard_normal((h, m)).astype(np.float32)
    x[:, ::5] = np.nan
    x[:, 1::7] = np.inf
    x[:, 2::9] = -np.inf
    x[:, 3::11] = -0.0
    x[:, 4::11] = 0.0
    x[:, 5::13] = 1e-42
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,kv_heads,d,page,keep,recent,sums", [
    ([100], 2, 64, 16, 60, 10, _heavy),
    ([1, 2, 3], 3, 16, 16, 2, 1, _heavy),
    ([5000, 17, 0, 2999, 3000, 3001], 2, 64, 64, 3000, 200, _heavy),
    ([700, 300], 2, 128, 20, 255, 0, _ties),
    ([700], 1, 16, 7, 257, 257, _heavy),
    ([900, 65], 2, 80, 48, 64, 3, _odd),
    ([4097], 1, 256, 1, 1, 0, _ties),
    ([2000], 2, 32, 128, 1999, 1000, _ties),
    ([16385, 12000], 1, 16, 64, 5000, 77, _heavy),
    ([40000], 1, 16, 64, 39990, 5, _ties),
    ([65537], 1, 16, 128, 30001, 1, _odd),
])
def test_eviction(dtype, lengths, kv_heads, d, page, keep, recent, sums):
    check_eviction(dtype, lengths, kv_heads, d, page, keep, recent, sums)


def test_eviction_into_pages_of_another_size():
    check_eviction("bf16", [500, 90], 2, 64, 16, 128, 32, _heavy, into_page=48, more_pages=1)


def test_eviction_within_one_pool():
    """K, V and lengths of both caches are the same arrays; the pages are others."""
    p = Problem("bf16", [(0, 90), (0, 40)], 2, 2, 64, 16, spare=6, garbage=False).on_gpu()
    free = sorted(set(range(p.pages)) - set(p.table.flatten().tolist()))[:6]
    table = torch.tensor(free, dtype=torch.int32, device="cuda").view(2, 3)
    into = attnw.AttnwCache(p.dev["K"], p.dev["V"], table, p.dev["lengths"], 2, p.pages, 3, 16, 2, 64, attnw.ATTNW_BF16)
    sums = torch.rand((2, 2, p.max_pages * 16), device="cuda")
    into_sums, kept = torch.zeros((2, 2, 48), device="cuda"), torch.zeros((2, 2, 41), dtype=torch.int32, device="cuda")
    attnw.attnw_cache_evict(p.cache, into, sums, into_sums, kept, 41, 8)
    torch.cuda.synchronize()
    want = evicted(sums.cpu().numpy(), [90, 40], 41, 8)
    assert np.array_equal(kept.cpu().numpy(), want) and p.dev["lengths"].tolist() == [41, 40]
    K = p.dev["K"].cpu()
    assert torch.equal(K[p.table.flatten().long()], p.K[p.table.flatten().long()]), "the pages that were there"
    for h in range(2):
        slot = torch.from_numpy(want[0, h].astype(np.int64))
        to = torch.arange(41)
        assert torch.equal(K[table[0].cpu().long()[to // 16], h, to % 16], p.K[p.table[0].long()[slot // 16], h, slot % 16])
