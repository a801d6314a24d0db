"""The example of serving from a paged cache: its layer against dense attention in 64 bits, tokens replayed from a recording, eviction in between."""
import importlib.util
import os

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")


@pytest.fixture(scope="module")
def example():
    require_gpu()
    spec = importlib.util.spec_from_file_location("paged_serving", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


class Dense:
    """One sequence of the layer in 64 bits: all its keys and values, which of them each kv head still has."""

    def __init__(self, layer, cap):
        self.layer, self.cap = layer, cap
        self.K, self.V = [], []
        self.has = [[] for _ in range(layer.kv_heads)]

    def forward(self, x):
        a, outs = self.layer, []
        H, Hk, d, half = a.heads, a.kv_heads, a.d, a.rot // 2
        for row in x.double().cpu():
            p = row @ a.w_in.double().cpu()
            position = len(self.K)
            angle = position * 10000.0 ** (-torch.arange(0, a.rot, 2, dtype=torch.float64) / a.rot)
            phase = torch.polar(torch.ones_like(angle), angle)

            def turn(v):
                z = torch.complex(v[..., :half], v[..., half:2 * half]) * phase
                return torch.cat([z.real, z.imag, v[..., 2 * half:]], -1)
            q, k = turn(p[:H * d].view(H, d)), turn(p[H * d:(H + Hk) * d].view(Hk, d))
            self.K.append(k)
            self.V.append(p[(H + Hk) * d:].view(Hk, d))
            O = []
            for h in range(H):
                g = h // (H // Hk)
                if h % (H // Hk) == 0:
                    self.has[g].append(position)
                keys = torch.stack([self.K[j][g] for j in self.has[g]])
                s = keys @ q[h] * d ** -0.5
                w = torch.softmax(self.cap * torch.tanh(s / self.cap), 0)
                O.append(w @ torch.stack([self.V[j][g] for j in self.has[g]]))
            outs.append(torch.cat(O) @ a.w_out.double().cpu())
        return torch.stack(outs)


# Projections and outputs are rounded to bf16 on the way (2^-8 each: queries, keys, values, weights, attention, layer output); outputs are sums of
# some hundred products of the size of 1: six roundings of the largest term's size, in the mean over a row far less.
def near(got, want):
    off = (got.double().cpu() - want).norm(dim=1) / want.norm(dim=1)
    assert float(off.max()) <= 6 * 2.0 ** -8, float(off.max())


def test_layer_against_dense_attention(example):
    torch.manual_seed(3)
    model, cap = 256, 20.0
    layer = example.PagedLayer(model, heads=4, kv_heads=2, d=64, batch=3, pages=60, max_pages=10, page_size=16, rot=32, positions=512, cap=cap)
    dense = [Dense(layer, cap) for _ in range(3)]
    x = [torch.randn((n, model), device="cuda").to(torch.bfloat16) for n in (70, 33, 5)]
    for at in (0, 32, 64):
        chunk = [p[at:at + 32] for p in x]
        for d, c, out in zip(dense, chunk, layer.prefill(chunk)):
            if c.shape[0]:
                near(out, d.forward(c))
    assert layer.lengths.tolist() == [70, 33, 5]
    # every token gave its heads' weights away: so many that the slots have together
    for b, n in enumerate((70, 33, 5)):
        assert abs(float(layer.sums[b].sum()) - n * 4) <= n * 4 * 1e-5
    kept = layer.evict(40, recent=8)
    assert layer.lengths.tolist() == [40, 33, 5] and len(layer.free) == 60 - 3 - 3 - 1
    for g in range(2):
        stay = kept[0, g].tolist()
        assert stay[-8:] == list(range(62, 70))
        dense[0].has[g] = stay
    step = layer.recorded_step()
    for _ in range(20):                           # (over the end of a page)
        token = torch.randn((3, model), device="cuda").to(torch.bfloat16)
        out = step(token)
        torch.cuda.synchronize()
        for b in range(3):
            near(out[b:b + 1], dense[b].forward(token[b:b + 1]))
    assert layer.lengths.tolist() == [60, 53, 25]
    layer.evict(50, recent=50)
    assert layer.lengths.tolist() == [50, 50, 25]


def test_the_example_runs(example, capsys):
    example.main()
    text = capsys.readouterr().out
    assert "slots after eviction down to 512: [512, 333, 64, 512]" in text and "slots after 32 tokens" in text


def test_a_recording_keeps_what_it_reads(example):
    """Small tensors made between the replays take no memory that the recording reads or writes: their contents stay, and the outputs are right."""
    torch.manual_seed(4)
    model, cap = 256, 20.0
    layer = example.PagedLayer(model, heads=4, kv_heads=2, d=64, batch=3, pages=60, max_pages=10, page_size=16, rot=32, positions=512, cap=cap)
    dense = [Dense(layer, cap) for _ in range(3)]
    x = [torch.randn((n, model), device="cuda").to(torch.bfloat16) for n in (40, 33, 5)]
    for d, c, out in zip(dense, x, layer.prefill(x)):
        near(out, d.forward(c))
    step = layer.recorded_step()
    others = []
    for i in range(6):
        for n in (1, 3, 4, 32, 128):              # up to 512 bytes: the sizes that starts and positions have
            others += [torch.full((n,), 400 + i, dtype=torch.int32, device="cuda") for _ in range(8)]
        token = torch.randn((3, model), device="cuda").to(torch.bfloat16)
        out = step(token)
        torch.cuda.synchronize()
        for b in range(3):
            near(out[b:b + 1], dense[b].forward(token[b:b + 1]))
    for k, other in enumerate(others):
        assert bool((other == 400 + k // 40).all()), f"tensor {k}, of {other.numel()} numbers, was written to"


def test_prompts_between_recorded_steps(example):
    """More of a prompt goes in between two replays: the next token's position follows it."""
    torch.manual_seed(5)
    model, cap = 256, 20.0
    layer = example.PagedLayer(model, heads=4, kv_heads=2, d=64, batch=2, pages=60, max_pages=10, page_size=16, rot=64, positions=512, cap=cap)
    dense = [Dense(layer, cap) for _ in range(2)]

    def prompt(*sizes):
        x = [torch.randn((n, model), device="cuda").to(torch.bfloat16) for n in sizes]
        for d, c, out in zip(dense, x, layer.prefill(x)):
            if c.shape[0]:
                near(out, d.forward(c))
    prompt(20, 7)
    step = layer.recorded_step()
    for sizes in ((0, 30), (17, 1)):
        for _ in range(2):
            token = torch.randn((2, model), device="cuda").to(torch.bfloat16)
            out = step(token)
            torch.cuda.synchronize()
            for b in range(2):
                near(out[b:b + 1], dense[b].forward(token[b:b + 1]))
        prompt(*sizes)
