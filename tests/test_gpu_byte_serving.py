"""Serving from a paged cache in 8 bits as a program does it: text and images by several axes, prompts in chunks, then tokens from a recording, in which appending
and attention follow each other; every call against the definitions on the host (byte_util, paged_util)."""
import pytest
import torch

import paper_2407_13885_amd as attnw
from byte_util import Problem8, appended, axis_map, same_bytes, turned32, values
from gpu_util import DT, TORCH_DT, require_gpu
from paged_util import within
from test_gpu_rotary import bound_of

pytestmark = pytest.mark.gpu

ROWS = 256                                        # of the table


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Server:
    """A cache of `batch` sequences with what the host knows of it: bytes, scales, lengths, and the position that each sequence's next token has."""

    def __init__(self, dtype, batch, heads, kv_heads, d, page, block, max_pages, pairs, order, layout, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.dtype, self.batch, self.heads, self.kv_heads, self.d, self.page, self.block, self.max_pages = dtype, batch, heads, kv_heads, d, page, block, max_pages
        self.pages = batch * max_pages + 2
        self.table = torch.randperm(self.pages, generator=self.g)[:batch * max_pages].to(torch.int32).view(batch, max_pages)
        self.lengths = torch.zeros(batch, dtype=torch.int32)
        shape = (self.pages, kv_heads, page, d)
        self.state = {n: (torch.full(shape, 0x7f, dtype=torch.uint8), torch.full((self.pages, kv_heads, page // block), 0xff, dtype=torch.uint8)) for n in "KV"}
        self.axes, self.layout, self.rot = attnw.AttnwAxes(pairs, order, True), layout, 2 * sum(pairs)
        self.axis_of = axis_map(pairs, order)[0]
        self.dev = {"table": self.table.cuda(), "lengths": self.lengths.cuda()}
        for n, (b, s) in self.state.items():
            self.dev[n], self.dev[n + "_scales"] = b.cuda(), s.cuda()
        self.angles = torch.empty((ROWS, self.rot), device="cuda")
        attnw.attnw_rotary_axes_table(self.angles, self.axes, ROWS, self.rot)
        self.cache = attnw.AttnwByteCache(self.dev["K"], self.dev["V"], self.dev["K_scales"], self.dev["V_scales"], self.dev["table"], self.dev["lengths"], batch,
                                          self.pages, max_pages, page, block, kv_heads, d, DT[dtype])
        self.rule = attnw.AttnwRule(d ** -0.5, 25.0)
        self.next = [0] * batch

    def positions(self, new, image):
        """[axes][tokens]: text stands at one place on all axes, an image's patches at its time and their rows and columns behind the text's."""
        n_axes, out = len(set(self.axis_of)), []
        for b, n in enumerate(new):
            p = torch.full((n_axes, n), self.next[b])
            if image and n >= 4:
                i = torch.arange(n)
                for a in range(1, n_axes):
                    p[a] += i // 3 if a % 2 else i % 3
                self.next[b] = int(p.max()) + 1
            else:
                p += torch.arange(n)
                self.next[b] += n
            out.append(p)
        return torch.cat(out, 1).to(torch.int32)

    def rows(self, tokens):
        x = torch.randn((tokens, (self.heads + 2 * self.kv_heads) * self.d), generator=self.g) * torch.exp2(2 * torch.randn((tokens, 1), generator=self.g))
        return x.to(TORCH_DT[self.dtype])

    def buffers(self, tokens):
        t = TORCH_DT[self.dtype]
        size = attnw.attnw_byte_paged_workspace(self.cache, tokens, self.heads)
        return {"x": torch.empty((tokens, (self.heads + 2 * self.kv_heads) * self.d), dtype=t, device="cuda"), "size": size,
                "positions": torch.empty((len(set(self.axis_of)), tokens), dtype=torch.int32, device="cuda"),
                "starts": torch.empty(self.batch + 1, dtype=torch.int32, device="cuda"), "R": torch.empty((tokens, self.heads, self.d), dtype=t, device="cuda"),
                "O": torch.empty((tokens, self.heads, self.d), dtype=t, device="cuda"), "lse": torch.empty((tokens, self.heads), device="cuda"),
                "work": torch.empty(max(16, size), dtype=torch.uint8, device="cuda")}

    def call(self, to, tokens, stream=None):
        wide, x = to["x"].shape[1], to["x"]
        keys = x[:, self.heads * self.d:]
        attnw.attnw_byte_cache_append(self.cache, x, keys, keys[:, self.kv_heads * self.d:], to["R"], self.angles, to["positions"], self.axes, to["starts"], tokens,
                                      self.heads, self.rot, ROWS, wide, wide, self.layout, stream)
        attnw.attnw_byte_paged_attention(self.cache, self.rule, to["R"], to["O"], to["lse"], to["starts"], tokens, self.heads, self.heads * self.d, to["work"],
                                         to["size"], stream)

    def check(self, new, x, positions, to):
        """What the calls left, against the definitions: bytes and scales exactly, queries, outputs and lse by their bounds."""
        T, wide = sum(new), self.heads * self.d
        starts = torch.tensor([sum(new[:b]) for b in range(self.batch + 1)], dtype=torch.int32)
        self.lengths += torch.tensor(new, dtype=torch.int32)
        q, k, v = x.split([wide, self.kv_heads * self.d, self.kv_heads * self.d], 1)
        table = self.angles.cpu()
        k32 = turned32(k.reshape(T, self.kv_heads, self.d), table, positions, self.axis_of, self.rot, self.layout)
        for n, rows in (("K", k32), ("V", v.reshape(T, self.kv_heads, self.d).float())):
            self.state[n] = appended(*self.state[n], self.block, self.table, self.lengths, starts, self.page, rows)
            same_bytes(self.dev[n], self.state[n][0], n)
            assert torch.equal(self.dev[n + "_scales"].cpu(), self.state[n][1]), n + "_scales"
        assert torch.equal(self.dev["lengths"].cpu(), self.lengths)
        q = q.reshape(T, self.heads, self.d)
        within(to["R"], turned32(q, table, positions, self.axis_of, self.rot, self.layout).double(), 2 * bound_of(q, self.dtype), "R")
        p = Problem8.__new__(Problem8)            # the attention of these very queries over these very bytes
        p.dtype, p.sequences, p.heads, p.kv_heads, p.d, p.page = self.dtype, list(zip(new, self.lengths.tolist())), self.heads, self.kv_heads, self.d, self.page
        p.batch, p.T, p.group, p.table, p.starts = self.batch, T, self.heads // self.kv_heads, self.table, starts
        p.Q, p.scale, p.cap, p.window, p.prefix, p.slopes = to["R"].cpu().flatten(1), self.d ** -0.5, 25.0, 0, None, None
        p.K, p.V = (values(*self.state[n], self.block) for n in "KV")
        O, lse, O_off, lse_off = p.attention()
        within(to["O"], O, O_off, "O")
        within(to["lse"], lse, lse_off, "lse")

    def chunk(self, new, image=False):
        x, positions, to = self.rows(sum(new)), self.positions(new, image), self.buffers(sum(new))
        to["x"].copy_(x)
        to["positions"].copy_(positions)
        to["starts"].copy_(torch.tensor([sum(new[:b]) for b in range(self.batch + 1)], dtype=torch.int32))
        self.dev["lengths"].add_(torch.tensor(new, dtype=torch.int32, device="cuda"))
        self.call(to, sum(new), torch.cuda.current_stream())
        self.check(new, x, positions, to)

    def recorded(self, new, work=None):
        """A step of so many tokens a sequence, recorded: all that it reads and writes."""
        to = self.buffers(sum(new))
        if work is not None:
            assert work.numel() >= to["size"]
            to["work"] = work
        to["starts"].copy_(torch.tensor([sum(new[:b]) for b in range(self.batch + 1)], dtype=torch.int32))
        to["more"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            self.dev["lengths"].add_(to["more"])
            self.call(to, sum(new), torch.cuda.current_stream())
        return graph, to

    def step(self, recording, new):
        graph, to = recording
        x, positions = self.rows(sum(new)), self.positions(new, False)
        to["x"].copy_(x)
        to["positions"].copy_(positions)
        to["O"].fill_(7.0)
        to["work"].fill_(0xff)                    # (of any content)
        graph.replay()
        torch.cuda.synchronize()
        self.check(new, x, positions, to)


def server(dtype, **more):
    sizes = dict(batch=3, heads=8, kv_heads=2, d=64, page=16, block=8, max_pages=12, pairs=[8, 10, 10], order=attnw.ATTNW_TURNS, layout=attnw.ATTNW_HALVES, seed=1)
    sizes.update(more)
    return Server(dtype, **sizes)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("more", [{}, dict(order=attnw.ATTNW_SECTIONS, layout=attnw.ATTNW_PAIRS, pairs=[16, 8], block=16), dict(d=144, heads=3, kv_heads=3, pairs=[72], page=10, block=5)],
                         ids=["turns", "sections", "one axis"])
def test_prompts_and_recorded_tokens(dtype, more):
    s = server(dtype, **more)
    for new, image in (((20, 7, 0), False), ((33, 0, 12), True), ((1, 30, 9), True)):
        s.chunk(list(new), image)
    step = s.recorded([1, 1, 1])
    for i in range(7):                            # (over the ends of blocks and of a page)
        s.step(step, [1, 1, 1])
        if i == 3:
            s.chunk([5, 0, 2])                    # more of a prompt between two replays


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_recordings_share_a_workspace(dtype):
    """Tokens one by one and drafts of several, each recorded: replayed in turns on one stream, with one workspace."""
    s = server(dtype, seed=2)
    s.chunk([40, 3, 21])
    one, many = [1, 1, 1], [3, 4, 2]
    work = torch.empty(max(attnw.attnw_byte_paged_workspace(s.cache, n, s.heads) for n in (3, 9)), dtype=torch.uint8, device="cuda")
    recordings = {1: (s.recorded(one, work), one), 2: (s.recorded(many, work), many)}
    for which in (1, 2, 2, 1, 2, 1, 1):
        s.step(*recordings[which])


def test_drafts_that_are_rejected():
    """Lengths go back over tokens that are not taken: what is appended later takes their slots, a block's scale stays at least what it was."""
    s = server("bf16", seed=3)
    s.chunk([18, 5, 30])
    for taken in ([1, 0, 3], [4, 2, 0], [2, 2, 2]):
        s.chunk([4, 4, 4])
        s.lengths += torch.tensor(taken, dtype=torch.int32) - 4
        s.dev["lengths"].copy_(s.lengths)
        s.next = [n - 4 + t for n, t in zip(s.next, taken)]
    s.chunk([1, 1, 1])


@pytest.mark.parametrize("layout", [attnw.ATTNW_HALVES, attnw.ATTNW_PAIRS])
def test_rotary_axes_recorded(layout):
    """Turned and back, recorded: every replay as the calls outside one, whatever the positions are by then."""
    axes, tokens, heads, d = attnw.AttnwAxes([10, 11, 11], attnw.ATTNW_TURNS), 77, 5, 80
    table = torch.empty((ROWS, 64), device="cuda")
    attnw.attnw_rotary_axes_table(table, axes, ROWS, 64)
    x = torch.empty((tokens, heads * d), dtype=torch.bfloat16, device="cuda")
    positions = torch.zeros((3, tokens), dtype=torch.int32, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def both(y, dx, stream):
        for a, b, back in ((x, y, 0), (y, dx, 1)):
            attnw.attnw_rotary_axes(a, b, table, positions, axes, tokens, heads, d, 64, ROWS, heads * d, heads * d, layout, back, attnw.ATTNW_BF16, stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        both(y, dx, torch.cuda.current_stream())
    g = torch.Generator().manual_seed(4)
    for _ in range(4):
        x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        positions.copy_(torch.randint(0, ROWS, positions.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(y), torch.empty_like(dx)
        both(*want, torch.cuda.current_stream())
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
