"""fp32 attention over a paged cache in 8 bits by blocks of 128 rows (d = 80, 96 and above 128): every rule, and what test_gpu_byte_attention asks of both kernels at head
sizes that go by blocks of 16 rows in any case."""
import pytest
import torch

import paper_2407_13885_amd as attnw
from byte_util import Problem8
from gpu_util import kernels, require_gpu
from paged_util import within
from test_gpu_byte_attention import check
from test_gpu_paged import RULES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(autouse=True)
def _blocks(monkeypatch):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", "tiles")


def kernel_of(p):
    size, d = attnw.attnw_byte_paged_workspace(p.cache, p.T, p.heads), p.dev
    O, work = torch.empty((p.T, p.heads, p.d), device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda")
    return kernels(lambda s: attnw.attnw_byte_paged_attention(p.cache, p.rule, d["Q"], O, None, d["starts"], p.T, p.heads, p.q_stride, work, size, s))[0]


@pytest.mark.parametrize("more", [{}, dict(cap=20.0), dict(slopes=True), dict(cap=20.0, slopes=True)], ids=["plain", "cap", "bias", "both"])
@pytest.mark.parametrize("d", range(16, 257, 16))
def test_which_kernel(d, more, monkeypatch):
    p = Problem8("f32", [(1, 60), (9, 9)], 4, 2, d, 16, 8, **more).on_gpu()
    assert ("paged_tiles_kernel" if d in (80, 96) or d > 128 else "byte_rows_kernel") in kernel_of(p)
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", "rows")
    assert "byte_rows_kernel" in kernel_of(p)


def test_a_chunk_goes_there_by_itself(monkeypatch):
    monkeypatch.delenv("ATTNW_PAGED_KERNEL")
    for d in (96, 160):
        assert "paged_tiles_kernel" in kernel_of(Problem8("f32", [(256, 300)], 8, 2, d, 16, 8).on_gpu())


# sequences (new, in use), heads, kv heads, page, block
SHAPES = [
    ("one token alone", [(1, 1)], 1, 1, 16, 16),
    ("tokens of several lengths, some empty", [(1, 1), (0, 40), (1, 33), (1, 640), (0, 0), (1, 129)], 8, 4, 32, 32),
    ("a chunk at the start", [(37, 37)], 4, 4, 16, 4),
    ("a chunk over others", [(65, 300), (3, 259), (128, 128)], 8, 2, 20, 10),
    ("groups that blocks cut", [(19, 90), (5, 5), (50, 50)], 21, 3, 7, 7),
    ("more heads than a block has rows", [(2, 70), (1, 213)], 140, 1, 64, 64),
    ("a scale for every slot", [(4, 101), (70, 333)], 2, 1, 5, 1),
    ("more places than are kept on chip", [(2, 1300)], 2, 1, 1, 1),
    ("many sequences", [(i % 3, i % 3 + 7 * i % 60) for i in range(150)], 4, 2, 16, 8),
]


@pytest.mark.parametrize("d", [80, 96, 160, 192, 256])
@pytest.mark.parametrize("name,sequences,heads,kv_heads,page,block", SHAPES, ids=[s[0] for s in SHAPES])
def test_attention(d, name, sequences, heads, kv_heads, page, block):
    check(Problem8("f32", sequences, heads, kv_heads, d, page, block, seed=d))


@pytest.mark.parametrize("d", [80, 96, 144, 176, 240])
@pytest.mark.parametrize("name,more", RULES, ids=[r[0] for r in RULES])
def test_rules(d, name, more):
    check(Problem8("f32", [(1, 410), (40, 333), (150, 420)], 8, 4, d, 32, 16, seed=d, **more))


@pytest.mark.parametrize("d", [96, 160, 224])
@pytest.mark.parametrize("more", [dict(cap=20.0), dict(cap=9.0, slopes=True), dict(slopes=True), dict(prefix=[1100]), dict(window=900), dict(window=200, prefix=[300], cap=40.0, slopes=True)],
                         ids=["cap", "both", "bias", "prefix", "window", "all"])
def test_long_runs(d, more):
    for m, block in ((1290, 16), (1322, 2)):
        check(Problem8("f32", [(70, m)], 2, 1, d, 32, block, seed=m, **more))


@pytest.mark.parametrize("d", [80, 160, 208])
@pytest.mark.parametrize("scale", [-0.125, 0.0, 3.0])
@pytest.mark.parametrize("more", [{}, dict(cap=30.0)], ids=["plain", "cap"])
def test_scales_of_either_sign(d, scale, more):
    p = Problem8("f32", [(1, 90), (20, 333)], 4, 2, d, 16, 16, seed=12, **more)
    p.scale = scale
    O, lse = p.on_gpu().run_attention()
    p.scale = abs(scale)
    if scale < 0:
        p.Q = -p.Q
    want, want_lse, off, lse_off = p.attention()
    within(O[:p.T], want, off, "O")
    within(lse[:p.T], want_lse, lse_off, "lse")


@pytest.mark.parametrize("d", [80, 160, 256])
def test_rows_that_see_nothing(d):
    """A sequence of more tokens than slots: those before its first slot see nothing."""
    p = Problem8("f32", [(4, 60)], 4, 2, d, 16, more_pages=1)
    p.lengths[0] = 2
    O, lse = p.on_gpu().run_attention()
    assert bool((O[:2] == 0).all()) and bool(torch.isneginf(lse[:2]).all())
    p.sequences, p.starts, p.T, p.Q, p.batch = [(2, 2)], torch.tensor([0, 2], dtype=torch.int32), 2, p.Q[2:], 1
    want, want_lse, off, lse_off = p.attention()
    within(O[2:], want, off, "O")
    within(lse[2:], want_lse, lse_off, "lse")
    O, lse = Problem8("f32", [(3, 0)], 4, 2, d, 16, more_pages=1).on_gpu().run_attention()       # no slot at all
    assert bool((O == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("d", [96, 160])
def test_scales_at_their_ends(d):
    p = Problem8("f32", [(5, 120), (33, 64)], 4, 2, d, 16, 4, seed=11)
    p.V_scales[p.table[0, 2].long()] = 127 - 117
    p.K_scales[p.table[0, 3].long()] = 127 - 117
    check(p.restate())
    p.V_scales[p.table[0, :4].long()] = 127 + 100
    check(p.restate())


def test_queries_in_wider_rows():
    p = Problem8("f32", [(3, 50), (90, 170)], 4, 2, 160, 16, 16, seed=13, q_pad=72)
    O, lse = check(p)
    assert O.shape[0] == p.T
