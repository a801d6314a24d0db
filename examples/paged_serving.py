"""An attention layer that serves from a paged cache: prompts of uneven length go in by chunks, tokens follow one by one (recorded once, replayed),
and sequences that outgrow their budget give up the slots that collected the least weight.  (Windows and slopes count slots: after that they are no
longer distances of positions, which the rotation keeps.)

    python examples/paged_serving.py

Random weights, bf16; torch makes the projections, everything between them and the output projection is the library's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_13885_amd as attnw  # noqa: E402


class PagedLayer:
    """One layer with its pool of pages.  `rot` columns of a head turn; `rule` as in attnw_rule (scale apart)."""

    def __init__(self, model, heads, kv_heads, d, batch, pages, max_pages, page_size, rot, positions=32768, seed=0, **rule):
        self.heads, self.kv_heads, self.d, self.batch, self.page_size, self.max_pages, self.rot = heads, kv_heads, d, batch, page_size, max_pages, rot
        g = torch.Generator(device="cuda").manual_seed(seed)
        wide = (heads + 2 * kv_heads) * d
        self.w_in = (torch.randn((model, wide), generator=g, device="cuda") * model ** -0.5).to(torch.bfloat16)
        self.w_out = (torch.randn((heads * d, model), generator=g, device="cuda") * (heads * d) ** -0.5).to(torch.bfloat16)
        shape = (pages, kv_heads, page_size, d)
        self.K, self.V = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.table = torch.zeros((batch, max_pages), dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.sums = torch.zeros((batch, kv_heads, max_pages * page_size), device="cuda")
        self.rows = positions
        self.angles = torch.empty((positions, rot), device="cuda")
        attnw.attnw_rotary_table(self.angles, positions, rot, stream=torch.cuda.current_stream())
        self.cache = self._cache(self.table)
        self.rule = attnw.AttnwRule(d ** -0.5, **rule)
        # the host's side: which pages are free, which a sequence has, how long it is, the position of its next token
        self.free = list(range(pages))
        self.owned = [[] for _ in range(batch)]
        self.in_use = [0] * batch
        self.next_position = [0] * batch

    def _cache(self, table):
        return attnw.AttnwCache(self.K, self.V, table, self.lengths, self.batch, self.K.shape[0], self.max_pages, self.page_size, self.kv_heads, self.d,
                                attnw.ATTNW_BF16)

    def reserve(self, new):
        """Pages for so many more slots of each sequence."""
        for b, n in enumerate(new):
            while len(self.owned[b]) * self.page_size < self.in_use[b] + n:
                self.owned[b].append(self.free.pop())
        table = torch.zeros((self.batch, self.max_pages), dtype=torch.int32)
        for b, pages in enumerate(self.owned):
            table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.table.copy_(table)

    def buffers(self, tokens):
        """What a call of so many tokens writes."""
        shape = (tokens, self.heads, self.d)
        size = attnw.attnw_paged_workspace(self.cache, tokens, self.heads)
        return {"R": torch.empty(shape, dtype=torch.bfloat16, device="cuda"), "O": torch.empty(shape, dtype=torch.bfloat16, device="cuda"),
                "lse": torch.empty(shape[:2], device="cuda"), "workspace": torch.empty(max(1, size), dtype=torch.uint8, device="cuda"), "bytes": size}

    def attend(self, projected, starts, positions, to):
        """Queries, keys and values of new tokens, the last slots of their sequences (lengths count them): into to["O"]."""
        stream, tokens, wide = torch.cuda.current_stream(), projected.shape[0], projected.shape[1]
        keys = projected[:, self.heads * self.d:]
        attnw.attnw_cache_append(self.cache, projected, keys, keys[:, self.kv_heads * self.d:], to["R"], self.angles, positions, starts, tokens, self.heads,
                                 self.rot, self.rows, wide, wide, attnw.ATTNW_HALVES, stream)
        attnw.attnw_paged_attention(self.cache, self.rule, to["R"], to["O"], to["lse"], starts, tokens, self.heads, self.heads * self.d, to["workspace"],
                                    to["bytes"], stream)
        attnw.attnw_paged_sums(self.cache, self.rule, to["R"], to["lse"], self.sums, self.sums, starts, tokens, self.heads, self.heads * self.d, stream)

    def prefill(self, xs):
        """Chunks of some sequences (xs[b] [n][model]); a list of outputs."""
        new = [x.shape[0] for x in xs]
        self.reserve(new)
        positions = torch.cat([torch.arange(p, p + n) for p, n in zip(self.next_position, new)]).to(torch.int32).cuda()
        starts = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        self.in_use = [m + n for m, n in zip(self.in_use, new)]
        self.next_position = [p + n for p, n in zip(self.next_position, new)]
        self.lengths.copy_(torch.tensor(self.in_use, dtype=torch.int32))
        buffers = self.buffers(sum(new))
        self.attend(torch.cat(xs) @ self.w_in, starts, positions, buffers)
        return list((buffers["O"].flatten(1) @ self.w_out).split(new))

    def recorded_step(self):
        """One token of every sequence: a function from x [batch][model] to the layer's output.  What lies between the projections is recorded once and
        replayed.  (Not the projections: a library's product may clear memory on its way in a form that a replay does not repeat.)"""
        starts = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda")
        positions = torch.zeros(self.batch, dtype=torch.int32, device="cuda")
        projected = torch.empty((self.batch, self.w_in.shape[1]), dtype=torch.bfloat16, device="cuda")
        buffers = self.buffers(self.batch)
        # (a recording holds addresses, not tensors: all that it reads and writes has to live as long as it does)
        buffers.update(starts=starts, positions=positions)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            self.lengths.add_(1)
            self.attend(projected, starts, positions, buffers)

        def step(x):
            self.reserve([1] * self.batch)
            self.in_use = [m + 1 for m in self.in_use]
            positions.copy_(torch.tensor(self.next_position, dtype=torch.int32))
            self.next_position = [p + 1 for p in self.next_position]
            projected.copy_(x @ self.w_in)
            graph.replay()
            return buffers["O"].flatten(1) @ self.w_out
        return step

    def evict(self, keep, recent):
        """Sequences of more than `keep` slots down to that; which slots stayed, [batch][kv_heads][keep]."""
        many = -(-keep // self.page_size)
        pages = [[self.free.pop() for _ in range(many)] for _ in range(self.batch)]
        table = torch.zeros((self.batch, self.max_pages), dtype=torch.int32)
        table[:, :many] = torch.tensor(pages, dtype=torch.int32)
        table = table.cuda()
        into = self._cache(table)
        sums = torch.zeros_like(self.sums)
        kept = torch.empty((self.batch, self.kv_heads, keep), dtype=torch.int32, device="cuda")
        attnw.attnw_cache_evict(self.cache, into, self.sums, sums, kept, keep, recent, torch.cuda.current_stream())
        self.table.copy_(table)
        self.sums.copy_(sums)
        for b in range(self.batch):               # (freed once the stream is past the call: what uses them next follows on it)
            self.free += self.owned[b]
            self.in_use[b] = min(self.in_use[b], keep)
            have = -(-self.in_use[b] // self.page_size)
            self.owned[b], spare = pages[b][:have], pages[b][have:]
            self.free += spare
        return kept


def main():
    torch.manual_seed(0)
    model, batch, page_size, budget = 1024, 4, 16, 512
    layer = PagedLayer(model, heads=16, kv_heads=4, d=64, batch=batch, pages=512, max_pages=64, page_size=page_size, rot=64, cap=30.0)
    prompts = [700, 333, 64, 512]
    x = [torch.randn((n, model), device="cuda").to(torch.bfloat16) for n in prompts]
    for at in range(0, max(prompts), 256):        # chunks of 256 tokens, what is left of each prompt
        layer.prefill([p[at:at + 256] for p in x])
    print("slots after the prompts:", layer.lengths.tolist(), "free pages:", len(layer.free))
    layer.evict(budget, recent=64)
    print(f"slots after eviction down to {budget}:", layer.lengths.tolist(), "free pages:", len(layer.free))
    token = torch.randn((batch, model), device="cuda").to(torch.bfloat16)
    step = layer.recorded_step()
    for i in range(32):
        out = step(token).float()
        token = (out / out.pow(2).mean(1, keepdim=True).sqrt()).to(torch.bfloat16)
        if max(layer.in_use) > budget + 24:
            layer.evict(budget, recent=64)
    torch.cuda.synchronize()
    print("slots after 32 tokens:", layer.lengths.tolist(), "free pages:", len(layer.free))
    print("weight that the first sequence's slots have collected, of all heads:", round(float(layer.sums[0, :, :layer.in_use[0]].sum()), 1))


if __name__ == "__main__":
    main()
