"""The paged cache in 8 bits stated on the host, and problems to compare on (with paged_util, whose definitions of attention hold for the values that it stands for)."""
import math

import numpy as np
import torch

import paper_2407_13885_amd as attnw
from gpu_util import DT, TORCH_DT
from paged_util import EPS, Problem

LEAST, MOST = -117, 119                           # exponents of a scale


def exponents(top):
    """The least e with top <= 448 * 2^e, in its range; top [...] in 64 bits, finite."""
    m, e = np.frexp(np.asarray(top, dtype=np.float64))        # 448 = 0.875 * 2^9
    return np.where(top > 0, np.clip(e - 9 + (m > 0.875), LEAST, MOST), LEAST).astype(np.int64)


def rounded(x, e):
    """x in units of 2^e (broadcast) as the bytes of e4m3 numbers, to nearest even; what is not finite as NaN."""
    y = torch.ldexp(x.double(), -torch.as_tensor(e).double()).float()         # (exact, but for what is far below the least number)
    y = torch.where(y.isfinite(), y.clamp(-448.0, 448.0), math.nan)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def numbers(b):
    return b.view(torch.float8_e4m3fn).float()


def held(x, block):
    """x [pages][kv_heads][page][d] as a cache holds it: bytes, and the bytes of the scales."""
    pages, heads, page, d = x.shape
    e = exponents(torch.nan_to_num(x.double().abs(), 0.0, 0.0).view(pages, heads, page // block, block * d).amax(-1).numpy())
    by_slot = torch.from_numpy(e).repeat_interleave(block, 2)[..., None]
    return rounded(x, by_slot), torch.from_numpy(e + 127).to(torch.uint8)


def values(b, scales, block):
    """What bytes and scales stand for, in fp32 (exact for scales from 2^-117 to 2^119)."""
    s = torch.ldexp(torch.ones(()), scales.clamp(1, 246).int() - 127).repeat_interleave(block, 2)
    return numbers(b) * s[..., None]


def is_nan(b):
    return (b & 0x7f) == 0x7f


class Problem8(Problem):
    """A ragged batch over a cache in 8 bits.  K and V of Problem are the values that the bytes K8, V8 and scales stand for."""

    def __init__(self, dtype, sequences, heads, kv_heads, d, page, block=None, spread=2.0, **more):
        garbage = more.pop("garbage", True)
        super().__init__(dtype, sequences, heads, kv_heads, d, page, garbage=False, **more)
        self.block = page if block is None else block
        g = torch.Generator().manual_seed(more.get("seed", 0) + 77)
        used = torch.zeros((self.pages, page), dtype=torch.bool)
        for b, (_, m) in enumerate(sequences):
            for j in range(m):
                used[self.table[b, j // page].long(), j % page] = True
        for name in ("K", "V"):
            x = getattr(self, name).float()
            x = x * torch.exp2(spread * (2 * torch.rand((self.pages, kv_heads, page // self.block, 1), generator=g) - 1)).repeat_interleave(self.block, 2)
            b, s = held(x, self.block)
            if garbage:                           # what no sequence has in use may hold anything, scales of blocks without such slots too
                b = torch.where(used[:, None, :, None], b, torch.randint(0, 256, b.shape, generator=g, dtype=torch.uint8) | 0x7f)
                some = used.view(self.pages, page // self.block, self.block).any(-1)
                s = torch.where(some[:, None], s, torch.randint(0, 256, s.shape, generator=g, dtype=torch.uint8))
            setattr(self, name + "8", b)
            setattr(self, name + "_scales", s)
        self.restate()

    def restate(self):
        """K and V by the bytes (after a change to them)."""
        self.K, self.V = values(self.K8, self.K_scales, self.block), values(self.V8, self.V_scales, self.block)
        return self

    def on_gpu(self):
        self.dev = {k: v.cuda() for k, v in vars(self).items() if isinstance(v, torch.Tensor) and k not in ("K", "V")}
        d = self.dev
        self.cache = attnw.AttnwByteCache(d["K8"], d["V8"], d["K_scales"], d["V_scales"], d["table"], d["lengths"], self.batch, self.pages, self.max_pages, self.page,
                                       self.block, self.kv_heads, self.d, DT[self.dtype])
        self.rule = attnw.AttnwRule(self.scale, self.cap, d.get("slopes"), d.get("prefix"), self.window)
        return self

    def attention(self):
        """As Problem's; fp32 products and sums run over three parts of one factor: three times the terms."""
        O, lse, O_off, lse_off = super().attention()
        return (O, lse, O_off, lse_off) if self.dtype == "bf16" else (O, lse, 3 * O_off, 3 * lse_off)

    def run_attention(self, stream=None):
        d = self.dev
        O = torch.full((max(1, self.T), self.heads, self.d), 7.0, dtype=TORCH_DT[self.dtype], device="cuda")
        lse = torch.full((max(1, self.T), self.heads), 7.0, device="cuda")
        size = attnw.attnw_byte_paged_workspace(self.cache, self.T, self.heads)
        work = torch.full((size + 1024,), 0xff, dtype=torch.uint8, device="cuda")   # NaN everywhere
        attnw.attnw_byte_paged_attention(self.cache, self.rule, d["Q"], O, lse, d["starts"], self.T, self.heads, self.q_stride, work, size, stream)
        torch.cuda.synchronize()
        assert bool((work[size:] == 0xff).all()), "written behind the workspace"
        return O, lse


def turned32(x, table, positions, axis_of, rot, layout):
    """x [T][heads][d] in fp32, its pairs turned by the definition's three roundings; positions [axes][T]."""
    x = x.float().clone()
    if not rot:
        return x
    at = positions.long()[torch.as_tensor(axis_of)].t()                       # [T][pairs]
    pair = torch.arange(rot // 2)
    known = (at >= 0) & (at < table.shape[0])
    at = at.clamp(0, table.shape[0] - 1)
    nan = torch.tensor(math.nan)
    c, s = torch.where(known, table[at, pair], nan)[:, None], torch.where(known, table[at, pair + rot // 2], nan)[:, None]
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == attnw.ATTNW_HALVES else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = x[..., one].clone(), x[..., two].clone()
    x[..., one], x[..., two] = a * c - b * s, b * c + a * s
    return x


def axis_map(pairs, order):
    """Axis and index of every pair."""
    if order == attnw.ATTNW_SECTIONS:
        return [a for a, n in enumerate(pairs) for _ in range(n)], [i for n in pairs for i in range(n)]
    axis, index, given = [], [], [0] * len(pairs)
    while len(axis) < sum(pairs):
        for a, n in enumerate(pairs):
            if given[a] < n:
                axis.append(a)
                index.append(given[a])
                given[a] += 1
    return axis, index


def appended(b, scales, block, table, lengths, starts, page, rows):
    """Bytes and scales after the new tokens' rows [T][kv_heads][d] in fp32 went in; the arguments stay as they are."""
    b, scales = b.clone(), scales.clone()
    pages, heads = b.shape[:2]
    slots = table.shape[1] * page
    for s in range(table.shape[0]):
        n, m = int(starts[s + 1] - starts[s]), min(max(int(lengths[s]), 0), slots)
        base = max(0, m - n)
        for slot0 in range(base // block * block, m if n else 0, block):
            first, last = max(slot0, base), min(slot0 + block, m)
            if last <= first:
                continue
            id, row = int(table[s, slot0 // page]), slot0 % page
            if not 0 <= id < pages:
                continue
            t = int(starts[s]) + n - (m - first)
            new = rows[t:t + last - first]                                    # [new][kv_heads][d]
            e = exponents(torch.where(new.isfinite(), new, 0.0).double().abs().amax((0, 2)).numpy())
            if first > slot0:
                old = np.clip(scales[id, :, row // block].numpy().astype(np.int64) - 127, LEAST, MOST)
                e = np.maximum(e, old)
                grown = torch.from_numpy(e - old)[:, None, None]
                rows_before = b[id, :, row:row + first - slot0]
                b[id, :, row:row + first - slot0] = torch.where(grown > 0, rounded(numbers(rows_before.contiguous()), grown), rows_before)
            scales[id, :, row // block] = torch.from_numpy(e + 127).to(torch.uint8)
            b[id, :, row + first - slot0:row + last - slot0] = rounded(new.transpose(0, 1), torch.from_numpy(e)[:, None, None])
    return b, scales


def same_bytes(got, want, what):
    got = got.cpu()
    bad = (got != want) & ~(is_nan(got) & is_nan(want))
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} bytes differ, the first at {at}: got {int(got[at])}, want {int(want[at])}")
