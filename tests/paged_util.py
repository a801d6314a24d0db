"""The paged cache and what works on it, stated in 64 bits on the host, and problems to compare on.

Everything is a loop over the definitions: slot j of sequence b is row j % page_size of page table[b][j // page_size]; a sequence's new tokens
are its last slots; a token at slot i sees j <= i, of those the last `window`, and every slot below the prefix.
"""
import math

import numpy as np
import torch

import paper_2407_13885_amd as attnw
from gpu_util import DT, TORCH_DT

EPS = 2.0 ** -24                                  # half a unit in the last place of fp32


class Problem:
    """A ragged batch over a cache.  sequences: (new tokens, slots in use) of each; every array a torch tensor on the host."""

    def __init__(self, dtype, sequences, heads, kv_heads, d, page, seed=0, spare=3, more_pages=0, cap=0.0, window=0, prefix=None, slopes=False,
                 sharp=1.0, garbage=True, q_pad=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.sequences, self.heads, self.kv_heads, self.d, self.page = dtype, sequences, heads, kv_heads, d, page
        self.batch, self.T = len(sequences), sum(n for n, _ in sequences)
        self.group = heads // kv_heads
        self.max_pages = max(1, max(-(-m // page) for _, m in sequences)) + more_pages
        self.pages = self.batch * self.max_pages + spare
        self.table = torch.randperm(self.pages, generator=g)[:self.batch * self.max_pages].to(torch.int32).view(self.batch, self.max_pages)
        self.lengths = torch.tensor([m for _, m in sequences], dtype=torch.int32)
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum([n for n, _ in sequences])]), dtype=torch.int32)
        t = TORCH_DT[dtype]
        shape = (self.pages, kv_heads, page, d)
        self.K = torch.randn(shape, generator=g).to(t)
        self.V = torch.randn(shape, generator=g).to(t)
        if garbage:                               # what no sequence has in use may hold anything
            used = torch.zeros((self.pages, page), dtype=torch.bool)
            for b, (_, m) in enumerate(sequences):
                for j in range(m):
                    used[self.table[b, j // page].long(), j % page] = True
            bad = torch.where(torch.rand((self.pages, 1, page, 1), generator=g) < 0.5, float("nan"), float("inf"))
            mask = ~used[:, None, :, None]
            self.K = torch.where(mask, bad.to(t), self.K)
            self.V = torch.where(mask, bad.to(t), self.V)
        self.q_stride = heads * d + q_pad
        self.Q = (sharp * torch.randn((max(1, self.T), self.q_stride), generator=g)).to(t)
        self.scale = float(np.float32(d ** -0.5))
        self.cap, self.window = float(np.float32(cap)), window
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int32)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, heads + 1) / heads).float() if slopes else None

    # ---- in 64 bits -----------------------------------------------------------------------------------------------------------------
    def rows(self, what, b, kv_head):
        """[slots in use][d] of sequence b."""
        m = self.sequences[b][1]
        ids = self.table[b, torch.arange(m) // self.page].long()
        return what[ids, kv_head, torch.arange(m) % self.page].double()

    def seen(self, b):
        """[new tokens][slots in use]"""
        n, m = self.sequences[b]
        i, j = torch.arange(m - n, m)[:, None], torch.arange(m)[None, :]
        s = j <= i
        if self.window:
            s = s & (j > i - self.window)
        if self.prefix is not None:
            s = s | (j < self.prefix[b])
        return s

    def query(self, b, h):
        n, first = self.sequences[b][0], int(self.starts[b])
        return self.Q[first:first + n, h * self.d:(h + 1) * self.d].double()

    def scores(self, b, h):
        """x [new tokens][slots], -inf where not seen, and how far fp32 may be off it."""
        n, m = self.sequences[b]
        q, k = self.query(b, h), self.rows(self.K, b, h // self.group)
        x = self.scale * (q @ k.t())
        # a sum of d products, the scale, the change to base 2 and the difference to the reference: each rounds once
        off = (self.d + 8) * EPS * self.scale * (q.abs() @ k.abs().t())
        if self.cap:
            x = self.cap * torch.tanh(x / self.cap)
            off = off + self.cap * 2.0 ** (-20 if self.dtype == "bf16" else -21)
        if self.slopes is not None:
            far = float(self.slopes[h]) * (torch.arange(m - n, m)[:, None] - torch.arange(m)[None, :]).abs().double()
            x = x - far
            off = off + 4 * EPS * (far + x.abs())
        return x.masked_fill(~self.seen(b), -math.inf), off + 4 * EPS * x.abs()

    def attention(self):
        """O, lse and the bounds of the two."""
        O, lse = torch.zeros((self.T, self.heads, self.d), dtype=torch.float64), torch.full((self.T, self.heads), -math.inf, dtype=torch.float64)
        O_off, lse_off = torch.zeros_like(O), torch.zeros_like(lse)
        for b, (n, m) in enumerate(self.sequences):
            if not n or not m:
                continue
            first = int(self.starts[b])
            for h in range(self.heads):
                x, off = self.scores(b, h)
                some = self.seen(b).any(1)
                l = torch.logsumexp(x, 1)
                w = torch.where(some[:, None], torch.exp(x - torch.where(some, l, 0.0)[:, None]), 0.0)
                v = torch.nan_to_num(self.rows(self.V, b, h // self.group))
                O[first:first + n, h] = w @ v
                lse[first:first + n, h] = l
                worst = torch.where(self.seen(b), off, 0.0).amax(1) if m else torch.zeros(n)
                # weights off by twice a score's error (theirs and their sum's), m sums; bf16 rounds weights and result, by up to 2^-8 each
                rel = 2.0 * worst + (m + 8) * EPS + (2.0 ** -7 if self.dtype == "bf16" else 0.0)
                O_off[first:first + n, h] = rel[:, None] * (w @ v.abs()) + 2.0 ** -120
                lse_off[first:first + n, h] = worst + (m + 8) * EPS + 2 * EPS * torch.where(some, l, 0.0).abs()
        return O, lse, O_off, lse_off

    def collected(self, lse, before):
        """sums [batch][kv_heads][slots a sequence can have] and their bound, from an lse [T][heads] in fp32."""
        slots = self.max_pages * self.page
        sums = torch.zeros((self.batch, self.kv_heads, slots), dtype=torch.float64)
        bound = torch.zeros_like(sums)
        for b, (n, m) in enumerate(self.sequences):
            if before is not None:
                sums[b, :, :m - n] = before[b, :, :m - n].double()
            first = int(self.starts[b])
            for h in range(self.heads if n and m else 0):
                x, off = self.scores(b, h)
                l = lse[first:first + n, h, None].double()
                w = torch.where(self.seen(b) & ~torch.isneginf(l), torch.exp(x - l), 0.0)
                sums[b, h // self.group, :m] += w.sum(0)
                bound[b, h // self.group, :m] += (w * (off + 4 * EPS * l.abs().nan_to_num(posinf=0.0) + (n * self.group + 8) * EPS)).sum(0)
            bound[b] += 8 * EPS * sums[b].abs() + 1e-30
        return sums, bound

    # ---- by the library -----------------------------------------------------------------------------------------------------------------
    def on_gpu(self):
        self.dev = {k: v.cuda() for k, v in vars(self).items() if isinstance(v, torch.Tensor)}
        d = self.dev
        self.cache = attnw.AttnwCache(d["K"], d["V"], d["table"], d["lengths"], self.batch, self.pages, self.max_pages, self.page, self.kv_heads,
                                      self.d, DT[self.dtype])
        self.rule = attnw.AttnwRule(self.scale, self.cap, d.get("slopes"), d.get("prefix"), self.window)
        return self

    def run_attention(self, stream=None):
        d = self.dev
        O = torch.full((max(1, self.T), self.heads, self.d), 7.0, dtype=TORCH_DT[self.dtype], device="cuda")
        lse = torch.full((max(1, self.T), self.heads), 7.0, device="cuda")
        size = attnw.attnw_paged_workspace(self.cache, self.T, self.heads)
        guard = 1024
        work = torch.full((size + guard,), 0xff, dtype=torch.uint8, device="cuda")   # NaN everywhere
        attnw.attnw_paged_attention(self.cache, self.rule, d["Q"], O, lse, d["starts"], self.T, self.heads, self.q_stride, work, size, stream)
        torch.cuda.synchronize()
        assert bool((work[size:] == 0xff).all()), "written behind the workspace"
        return O, lse

    def run_sums(self, lse, before, sums):
        attnw.attnw_paged_sums(self.cache, self.rule, self.dev["Q"], lse, before, sums, self.dev["starts"], self.T, self.heads, self.q_stride)
        torch.cuda.synchronize()
        return sums


def within(got, want, bound, what):
    got = got.detach().cpu().double()
    same = (got == want) | (torch.isneginf(got) & torch.isneginf(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound)
    if bool(bad.any()):
        at = np.unravel_index(int(torch.where(torch.isnan(off), math.inf, off / bound.clamp(min=1e-300)).argmax()), off.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond their bound, the worst at {tuple(int(i) for i in at)}: "
                             f"got {float(got[at])}, want {float(want[at])}, bound {float(bound[at]):.3e}")


def evicted(sums, lengths, keep, recent):
    """kept [batch][kv_heads][keep] by sorting."""
    batch, heads = sums.shape[:2]
    kept = np.full((batch, heads, keep), -1, np.int32)
    for b in range(batch):
        m = int(lengths[b])
        for h in range(heads):
            if m <= keep:
                kept[b, h, :m] = np.arange(m)
                continue
            x = sums[b, h, :m - recent].astype(np.float64)
            x = np.where(np.isnan(x), -np.inf, x)
            nan = np.isnan(sums[b, h, :m - recent])
            order = sorted(range(m - recent), key=lambda j: (nan[j], -x[j], j))
            kept[b, h] = sorted(order[:keep - recent] + list(range(m - recent, m)))
    return kept
