"""What is timed of serving from a paged cache held in 8 bits, and of rotary positions with several axes: the rotation and its gradient, appending
to the cache with the rotation on the way, and attention over it.

``run`` computes each in its plain form (elementary torch operations in 32 bits) or, where ``own`` is true, by the library's entry points;
``exact`` states the same from the definitions in 64 bits.

The cache: K and V are [pages][kv_heads][page][d] of e4m3 numbers, K_scales and V_scales [pages][kv_heads][page / block] of bytes; a byte s
stands for 2^(s - 127) and belongs to ``block`` slots of a kv head.  ``table`` [batch][most] names the pages of a sequence, ``lengths`` counts its slots
in use.  A sequence's new tokens (rows starts[b] .. starts[b + 1] - 1 of a call) are its last slots.

Axes: pair j of a head turns by the position that its token has on axis_of[j]; positions are [axes][tokens].
"""
import math
import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_TABLE_ROWS = 32768
_LEAST, _MOST = -117, 119                         # of a scale's exponent


# ---- cases -----------------------------------------------------------------------------------------------------------------------

def _axes(dtype, tokens, heads, d, rot, pairs, layout, inverse, order="sections", fresh=False):
    """pairs: how many pairs of columns each axis has; order: an axis' pairs lie together, or the axes take them in turns; fresh: frequencies of its own for
    each axis."""
    return {"call": "axes", "dtype": dtype, "tokens": tokens, "heads": heads, "d": d, "rot": rot, "pairs": pairs, "order": order, "fresh": fresh,
            "layout": layout, "inverse": inverse}


def _paged(call, dtype, batch, heads, kv_heads, d, page, block, new, cached, spread, **more):
    """new, cached: the most new tokens and earlier slots of a sequence; a sequence has a share of either from 1 - spread to 1."""
    return {"call": call, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "block": block, "new": new,
            "cached": cached, "spread": spread, "rot": 0, "pairs": "", "order": "sections", "fresh": False, "layout": "half", "cap": 0.0, "window": 0,
            "prefix": 0, "slopes": False, **more}


def listed():
    cases = [
        # training on video: queries and keys of 16 frames of 32 x 32 turned by time, height and width where the projection left them
        ("axes-bf16-video", _axes("bf16", 16384, 16, 128, 128, "16,24,24", "half", False)),
        # the gradient of the same in full precision, three images of 24 x 24 and a token more: height and width with frequencies of their own
        ("axes-f32-image-gradient", _axes("f32", 3 * 577, 12, 64, 64, "16,16", "interleaved", True, fresh=True)),
        # a long mixed prompt, heads of 80, the three axes dealt the columns in turns
        ("axes-bf16-turns", _axes("bf16", 4099, 20, 80, 80, "14,13,13", "half", False, order="turns")),
        # a decoding step of eight sequences: one token each, into blocks that are partly full; the smallest call
        ("append-bf16-step", _paged("append", "bf16", 8, 16, 8, 128, 16, 16, 1, 4096, 0.5, rot=128)),
        # prompts of a batch going into the cache in chunks of uneven length, text and images
        ("append-bf16-chunk", _paged("append", "bf16", 6, 32, 8, 128, 64, 64, 2048, 4096, 0.6, rot=64, layout="interleaved", pairs="8,12,12")),
        # full precision, odd pages with a scale for every twelve slots, half of a head turned
        ("append-f32-ragged", _paged("append", "f32", 5, 8, 8, 80, 48, 12, 197, 1025, 0.7, rot=40)),
        # one token of one sequence against its 4096 earlier ones: latency, the keys to be spread over the chip
        ("attention-bf16-step", _paged("attention", "bf16", 1, 16, 8, 128, 16, 16, 1, 4096, 0.0)),
        # one token each of 64 sequences of very different lengths: the cache is read once
        ("attention-bf16-batch", _paged("attention", "bf16", 64, 32, 8, 128, 64, 64, 1, 16384, 0.95)),
        # five tokens proposed for each of 16 sequences and checked at once, scores capped, a window and the first tokens
        ("attention-bf16-draft", _paged("attention", "bf16", 16, 16, 4, 64, 32, 32, 5, 8192, 0.5, cap=30.0, window=4096, prefix=4)),
        # a chunk of a long prompt over what is cached of it: matrix products
        ("attention-bf16-chunk", _paged("attention", "bf16", 1, 32, 8, 128, 64, 64, 2048, 14336, 0.0)),
        # full precision, uneven chunks, a bias by distance, a window and a prefix that every token sees, a scale for every ten slots
        ("attention-f32-ragged", _paged("attention", "f32", 5, 8, 8, 80, 20, 10, 197, 1025, 0.7, window=700, prefix=37, slopes=True)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _lengths(case):
    """New tokens and slots in use of every sequence: of the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    new, total = [], []
    for b in range(case["batch"]):
        share = 1.0 if b == 0 else 1.0 - case["spread"] * rng.random()
        n = max(1, int(round(case["new"] * (1.0 if b == 0 else 1.0 - case["spread"] * rng.random()))))
        new.append(n)
        total.append(n + int(round(case["cached"] * share)))
    return new, total


def _visible(case):
    """(query, key) pairs that see each other, of one head."""
    new, total = _lengths(case)
    pairs = 0
    for n, length in zip(new, total):
        for i in range(n):
            at = length - n + i
            low = max(0, at + 1 - case["window"]) if case["window"] else 0
            first = min(case["prefix"], length)
            pairs += first + max(0, at + 1 - max(low, first))
    return pairs


def _row(case):
    """Elements between a token's queries and the next one's: queries, keys and values of a token lie together."""
    if case["call"] == "axes":
        return (case["heads"] + 4) * case["d"]
    return (case["heads"] + 2 * case["kv_heads"]) * case["d"]


def _parts(rng, whole, most):
    """A whole number as a text of up to `most` others that sum to it."""
    count = min(whole, rng.randrange(1, most + 1))
    cuts = sorted(rng.sample(range(1, whole), count - 1)) if count > 1 else []
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [whole]))


def draw(rng):
    call = rng.choice(["axes", "axes", "append", "append", "attention", "attention", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = _SIZE[dtype]
    layout, order, fresh = rng.choice(["half", "interleaved"]), rng.choice(["sections", "turns"]), rng.random() < 0.5
    if call == "axes":
        d = rng.choice([64, 64, 128, 128, 32, 256, 72, rng.randrange(2, 129) * 2])
        rot = rng.choice([d, d, max(2, d // 4 // 2 * 2), rng.randrange(1, d // 2 + 1) * 2])
        heads = rng.choice([1, 2, 8, 12, 16, 20, 32])
        return _axes(dtype, _spread(rng, 1, max(1, (1 << 26) // ((heads + 4) * d * size))), heads, d, rot, _parts(rng, rot // 2, 4), layout,
                     rng.random() < 0.5, order, fresh)
    d = rng.choice([64, 64, 128, 128, 128, 32, 256, rng.randrange(16, 257, 16)])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 4, 7, 8])
    page = rng.choice([16, 16, 32, 64, 64, 128, rng.randrange(1, 200)])
    block = rng.choice([b for b in range(1, page + 1) if page % b == 0] + [page])
    spread = rng.choice([0.0, 0.5, 0.95])
    if call == "append":
        rot = rng.choice([d, d, max(2, d // 4 // 2 * 2), rng.randrange(1, d // 2 + 1) * 2])
        new = rng.choice([1, _spread(rng, 1, 2048)])
        most = max(1, int((1 << 27) / (new * (heads + 2 * kv_heads) * d * size)))
        return _paged(call, dtype, _spread(rng, 1, min(64, most)), heads, kv_heads, d, page, block, new, _spread(rng, 1, 4096), spread, rot=rot,
                      layout=layout, order=order, fresh=fresh, pairs=rng.choice(["", _parts(rng, rot // 2, 3)]))
    cached = _spread(rng, 1, 16384)
    new = rng.choice([1, 1, _spread(rng, 2, 16), _spread(rng, 2, 2048)])
    bytes_most = (1 << 29) / ((cached + new) * kv_heads * d)
    flops_most = (1.5e11 if dtype == "bf16" else 5e10) / (4.0 * new * heads * (cached + new) * d)
    if flops_most < 1.0:
        new = max(1, int(new * flops_most))
        flops_most = 1.0
    more = {"cap": rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), "slopes": rng.random() < 0.25,
            "window": rng.choice([0, 0, 0, _spread(rng, 1, cached + new)]), "prefix": rng.choice([0, 0, 0, rng.randrange(0, cached + new + 1)])}
    return _paged(call, dtype, _spread(rng, 1, max(1, min(64, bytes_most, flops_most))), heads, kv_heads, d, page, block, new, cached, spread, **more)


# ---- inputs ----------------------------------------------------------------------------------------------------------------------

def _normal(generator, shape, dtype, sharp=False):
    x = torch.randn(shape, generator=generator, device="cuda", dtype=torch.float32)
    if sharp:   # every row times a factor of its own: flat and peaked rows side by side
        x *= 0.5 + 1.5 * torch.rand(shape[:-1] + (1,), generator=generator, device="cuda")
    return x.to(_TORCH[dtype])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _axis_of(case):
    """The axis of every pair, and which of its axis' pairs it is."""
    left = [int(n) for n in case["pairs"].split(",")] if case["pairs"] else [case["rot"] // 2]
    if case["order"] == "sections":
        return [a for a, n in enumerate(left) for _ in range(n)], [i for n in left for i in range(n)]
    axis, index, given = [], [], [0] * len(left)
    while len(axis) < sum(left):                  # in turns, axes that have all of theirs passed over
        for a, n in enumerate(left):
            if given[a] < n:
                axis.append(a)
                index.append(given[a])
                given[a] += 1
    return axis, index


def _angles(case):
    """cos and sin of every position a program may meet, made once: [rows][rot], the cosines first."""
    axis, index = _axis_of(case)
    pairs, rot = [axis.count(a) for a in range(max(axis) + 1)], case["rot"]
    exponent = [i / pairs[a] for a, i in zip(axis, index)] if case["fresh"] else [2 * j / rot for j in range(rot // 2)]
    frequency = 10000.0 ** -torch.tensor(exponent, dtype=torch.float64, device="cuda")
    angle = torch.arange(_TABLE_ROWS, dtype=torch.float64, device="cuda")[:, None] * frequency
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


def _grid(axes, at):
    """Positions [axes][tokens]: the last axes count through a grid of 32 x 32 .., the first one on from where the token stands."""
    rows = [at // 32 ** (axes - 1 - a) % (32 if a else _TABLE_ROWS) + (0 if axes == 1 else 11) for a in range(axes)]
    return torch.stack(rows).to(torch.int32).contiguous()


def _exponents(top):
    """The least e with top <= 448 * 2^e, in its range."""
    m, e = torch.frexp(top)                       # 448 = 0.875 * 2^9
    return torch.where(top > 0, e - 9 + (m > 0.875).int(), _LEAST).clamp(_LEAST, _MOST)


def _held(generator, case, pages):
    """Keys or values as a cache holds them: e4m3 numbers and the bytes of their scales.  Blocks differ in size by a factor of four, columns by another."""
    Hk, page, block, d = case["kv_heads"], case["page"], case["block"], case["d"]
    x = torch.randn((pages, Hk, page // block, block, d), generator=generator, device="cuda")
    x *= torch.exp2(2.0 * torch.rand((pages, Hk, page // block, 1, 1), generator=generator, device="cuda") - 1.0)
    x *= torch.exp2(2.0 * torch.rand((Hk, 1, 1, d), generator=generator, device="cuda") - 1.0)
    e = _exponents(x.abs().amax((3, 4)))
    numbers = torch.ldexp(x, -e[..., None, None]).to(torch.float8_e4m3fn)
    return numbers.view(pages, Hk, page, d), (e + 127).to(torch.uint8)


def prepare(case, seed):
    generator = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case)
    dtype = case["dtype"]
    if case["rot"]:
        state["angles"] = _angles(case)
        state["axis_of"] = torch.tensor(_axis_of(case)[0], device="cuda")
    axes = len(case["pairs"].split(",")) if case.get("pairs") else 1
    if case["call"] == "axes":
        T, row = case["tokens"], _row(case)
        first = torch.randint(0, 4096, (1,), generator=generator, device="cuda")
        state["positions"] = _grid(axes, torch.arange(T, device="cuda") + first)
        state["X"] = _normal(generator, (T, row), dtype)          # (the last columns are other projections of the token)
        state["Y"] = torch.zeros((T, case["heads"] * case["d"]), device="cuda", dtype=_TORCH[dtype])
        if own:
            _handles(state)
        return state
    B, H, page = case["batch"], case["heads"], case["page"]
    new, total = _lengths(case)
    T, most = sum(new), max(-(-n // page) for n in total)
    pages = B * most + 3
    table = torch.randperm(pages, generator=generator, device="cuda")[:B * most].to(torch.int32)   # in no order
    state.update(new_tokens=new, total=total, T=T, pages=pages, most=most, table=table.view(B, most).contiguous(), lengths=_ints(total))
    state["starts"] = _ints([sum(new[:b]) for b in range(B + 1)])
    state["K"], state["K_scales"] = _held(generator, case, pages)
    state["V"], state["V_scales"] = _held(generator, case, pages)
    if case["call"] == "append":
        state["projected"] = _normal(generator, (T, _row(case)), dtype, sharp=True)
        at = torch.cat([torch.arange(m - n, m, device="cuda") for n, m in zip(new, total)])
        state["positions"] = _grid(axes, at)
        state["R"] = torch.zeros((T, H, case["d"]), device="cuda", dtype=_TORCH[dtype])
    else:
        state["Q"] = _normal(generator, (T, H, case["d"]), dtype, sharp=True)
        state["slope"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H) if case["slopes"] else None
        state["first"] = _ints([min(case["prefix"], n) for n in total]) if case["prefix"] else None
        state["O"] = torch.zeros((T, H, case["d"]), device="cuda", dtype=_TORCH[dtype])
        state["lse"] = torch.zeros((T, H), device="cuda", dtype=torch.float32)
    if own:
        _handles(state)
    return state


def _handles(state):
    """What a program keeps beside its tensors: the cache, the axes, the rule of the scores, a workspace."""
    import paper_2407_13885_amd as attnw
    state["code"] = {"bf16": attnw.ATTNW_BF16, "f32": attnw.ATTNW_F32}[state["dtype"]]
    if state.get("pairs"):
        state["axes"] = attnw.AttnwAxes([int(n) for n in state["pairs"].split(",")], {"sections": attnw.ATTNW_SECTIONS, "turns": attnw.ATTNW_TURNS}[state["order"]],
                                        int(state["fresh"]))
    if state["call"] == "axes":
        return
    state["cache"] = attnw.AttnwByteCache(state["K"], state["V"], state["K_scales"], state["V_scales"], state["table"], state["lengths"], state["batch"],
                                       state["pages"], state["most"], state["page"], state["block"], state["kv_heads"], state["d"], state["code"])
    if state["call"] == "attention":
        state["rule"] = attnw.AttnwRule(state["d"] ** -0.5, state["cap"], state["slope"], state["first"], state["window"])
        state["bytes"] = attnw.attnw_byte_paged_workspace(state["cache"], state["T"], state["heads"])
        state["workspace"] = torch.empty(max(1, state["bytes"]), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _plain(state)


def _outputs(s):
    if s["call"] == "axes":
        return s["Y"]
    if s["call"] == "append":
        return s["R"], s["K"], s["K_scales"], s["V"], s["V_scales"]
    return s["O"], s["lse"]


def _own(s):
    import paper_2407_13885_amd as attnw
    stream = torch.cuda.current_stream()
    layout = int(s["layout"] == "interleaved")
    if s["call"] == "axes":
        attnw.attnw_rotary_axes(s["X"], s["Y"], s["angles"], s["positions"], s["axes"], s["tokens"], s["heads"], s["d"], s["rot"], _TABLE_ROWS, _row(s),
                                s["heads"] * s["d"], layout, int(s["inverse"]), s["code"], stream)
    elif s["call"] == "append":
        x, wide = s["projected"], s["heads"] * s["d"]
        attnw.attnw_byte_cache_append(s["cache"], x, x[:, wide:], x[:, wide + s["kv_heads"] * s["d"]:], s["R"], s["angles"], s["positions"], s.get("axes"),
                                  s["starts"], s["T"], s["heads"], s["rot"], _TABLE_ROWS, _row(s), _row(s), layout, stream)
    else:
        attnw.attnw_byte_paged_attention(s["cache"], s["rule"], s["Q"], s["O"], s["lse"], s["starts"], s["T"], s["heads"], s["heads"] * s["d"],
                                     s["workspace"], s["bytes"], stream)
    return _outputs(s)


def _turned(s, x, inverse=False):
    """x [T][heads][d], its pairs turned by the angles of their axes in 32 bits."""
    rot = s["rot"]
    at, pair = s["positions"].long()[s["axis_of"]].t(), torch.arange(rot // 2, device="cuda")   # [T][pairs]
    cos, sin = s["angles"][at, pair][:, None], s["angles"][at, pair + rot // 2][:, None]
    sin = -sin if inverse else sin
    x = x.float()
    turning, rest = x[..., :rot], x[..., rot:]
    if s["layout"] == "half":
        a, b = turning[..., :rot // 2], turning[..., rot // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = turning[..., 0::2], turning[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _rounded(x, e):
    """x / 2^e in e4m3, the largest number where it would be larger (no number where x is none)."""
    y = torch.ldexp(x, -e)
    return torch.where(x.isinf(), math.nan, y.clamp(-448.0, 448.0)).to(torch.float8_e4m3fn).view(torch.uint8)


def _lay(s, name, x, sequence, slot):
    """x [T][kv_heads][d] in 32 bits into the slots of its tokens: scales first, by all of a block's rows, then old rows of blocks that were partly
    full, then the new ones."""
    Hk, page, block = s["kv_heads"], s["page"], s["block"]
    held, scales = s[name].view(torch.uint8), s[name + "_scales"]
    flat = scales.permute(0, 2, 1).reshape(-1, Hk).int() - 127                       # [pages * blocks of a page][kv_heads]
    where = s["table"][sequence, slot // page].long()
    at = where * (page // block) + slot % page // block                              # the block of every token
    need = torch.full_like(flat, _LEAST).index_reduce_(0, at, _exponents(x.nan_to_num(0.0, 0.0, 0.0).abs().amax(-1)), "amax")
    base = s["lengths"].long() - s["starts"].long().diff()                           # the first new slot of every sequence
    older = base % block > 0                                                         # (its block has rows already)
    b = torch.arange(s["batch"], device="cuda")
    open_page, open_block = s["table"][b, (base // page).clamp(max=s["most"] - 1)].long(), base % page // block
    spot = open_page * (page // block) + open_block
    before = flat[spot]
    now = torch.where(older[:, None], torch.maximum(need[spot], before), need[spot])
    need[spot] = now
    rows = open_block[:, None] * block + torch.arange(block, device="cuda")          # [batch][block]
    heads = torch.arange(Hk, device="cuda")[None, :, None]
    old = held[open_page[:, None, None], heads, rows[:, None]]                       # [batch][kv_heads][block][d]
    again = _rounded(old.view(torch.float8_e4m3fn).float(), (now - before)[:, :, None, None])
    keep = torch.arange(block, device="cuda") < (base % block)[:, None]              # [batch][block]
    held[open_page[:, None, None], heads, rows[:, None]] = torch.where(keep[:, None, :, None], again, old)
    held[where, :, slot % page] = _rounded(x, need[at][..., None])
    touched = torch.zeros(flat.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, at, True)[:, None]
    scales.copy_((torch.where(touched, need, flat) + 127).to(torch.uint8).view(s["pages"], page // block, Hk).permute(0, 2, 1))


def _gathered(s, name, b):
    """[kv_heads][slots in use][d] of sequence b, in 32 bits."""
    n, page, block = s["total"][b], s["page"], s["block"]
    at = s["table"][b, :-(-n // page)].long()
    numbers = s[name].view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
    scale = torch.exp2(s[name + "_scales"][at].float() - 127.0).repeat_interleave(block, 2)
    return (numbers * scale[..., None]).transpose(0, 1).reshape(s["kv_heads"], -1, s["d"])[:, :n]


def _scores(s, b):
    """[kv_heads][group][new tokens][slots] of sequence b, -inf where a token does not see a slot."""
    n, length, Hk, d = s["new_tokens"][b], s["total"][b], s["kv_heads"], s["d"]
    group = s["heads"] // Hk
    at = sum(s["new_tokens"][:b])
    q = s["Q"][at:at + n].float().view(n, Hk, group, d).permute(1, 2, 0, 3).reshape(Hk, group * n, d)
    scores = torch.matmul(q, _gathered(s, "K", b).transpose(1, 2).contiguous()) * d ** -0.5
    if s["cap"]:
        scores = s["cap"] * torch.tanh(scores / s["cap"])
    query = torch.arange(length - n, length, device="cuda")[:, None]
    key = torch.arange(length, device="cuda")[None, :]
    scores = scores.view(Hk, group, n, length)
    if s["slope"] is not None:
        scores = scores - s["slope"].view(Hk, group, 1, 1) * (query - key).abs().float()
    seen = key <= query
    if s["window"]:
        seen = seen & (key > query - s["window"])
    if s["first"] is not None:
        seen = seen | (key < s["first"][b])
    return scores.masked_fill(~seen, float("-inf"))


def _plain(s):
    if s["call"] == "axes":
        x = s["X"][:, :s["heads"] * s["d"]].view(s["tokens"], s["heads"], s["d"])
        s["Y"].copy_(_turned(s, x, s["inverse"]).flatten(1))
        return _outputs(s)
    H, Hk, d, T = s["heads"], s["kv_heads"], s["d"], s["T"]
    if s["call"] == "append":
        q, k, v = (x.reshape(T, -1, d) for x in s["projected"].split([H * d, Hk * d, Hk * d], 1))
        s["R"].copy_(_turned(s, q))
        sequence = torch.bucketize(torch.arange(T, device="cuda"), s["starts"][1:].long(), right=True)
        slot = s["lengths"].long()[sequence] - s["starts"].long()[sequence + 1] + torch.arange(T, device="cuda")
        _lay(s, "K", _turned(s, k), sequence, slot)
        _lay(s, "V", v.float(), sequence, slot)
        return _outputs(s)
    at = 0
    for b, n in enumerate(s["new_tokens"]):
        scores = _scores(s, b)
        top = scores.amax(-1, keepdim=True)
        weights = torch.exp(scores - top)
        total = weights.sum(-1, keepdim=True)
        o = torch.matmul((weights / total).view(Hk, H // Hk * n, -1), _gathered(s, "V", b))
        s["O"][at:at + n] = o.view(H, n, d).transpose(0, 1)
        s["lse"][at:at + n] = (top + torch.log(total)).view(H, n).t()
        at += n
    return _outputs(s)


# ---- the bytes and operations that a pass cannot do without ------------------------------------------------------------------------

def work(case):
    size = _SIZE[case["dtype"]]
    axes = len(case["pairs"].split(",")) if case["pairs"] else 1
    if case["call"] == "axes":
        turned = case["tokens"] * case["heads"]
        return {"bytes": 2 * turned * case["d"] * size + case["tokens"] * 4 * (case["rot"] + axes), "flops": 3 * turned * case["rot"]}
    new, total = _lengths(case)
    T, H, Hk, d = sum(new), case["heads"], case["kv_heads"], case["d"]
    if case["call"] == "append":
        blocks = sum(-(-m // case["block"]) - (m - n) // case["block"] for n, m in zip(new, total))
        return {"bytes": T * (2 * H * d * size + 2 * Hk * d * (size + 1) + 4 * (case["rot"] + axes)) + 2 * blocks * Hk,
                "flops": 3 * T * (H + Hk) * case["rot"] + 4 * T * Hk * d}
    # slots that some new token sees
    read = sum(max(n, min(m, min(case["prefix"], m) + n + case["window"] - 1)) if case["window"] else m for n, m in zip(new, total))
    return {"bytes": 2 * read * Hk * (d + 1.0 / case["block"]) + T * H * (2 * d * size + 4), "flops": 4 * _visible(case) * H * d}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    wide = torch.float64

    def turn(x, inverse):                         # x [T][heads][d]: pairs as complex numbers times exp(i angle)
        rot = case["rot"]
        y = x.to(wide).clone()
        for j, a in enumerate(_axis_of(case)[0]):
            row = s["angles"][s["positions"][a].long()].to(wide)
            phase = torch.complex(row[:, j], -row[:, rot // 2 + j] if inverse else row[:, rot // 2 + j])[:, None]
            one, two = (j, rot // 2 + j) if case["layout"] == "half" else (2 * j, 2 * j + 1)
            z = torch.complex(y[..., one], y[..., two]) * phase
            y[..., one], y[..., two] = z.real, z.imag
        return y

    if case["call"] == "axes":
        return turn(s["X"][:, :case["heads"] * case["d"]].reshape(case["tokens"], case["heads"], case["d"]), case["inverse"]).flatten(1)
    B, H, Hk, d, page, block = case["batch"], case["heads"], case["kv_heads"], case["d"], case["page"], case["block"]
    slots = [torch.arange(m, device="cuda") for m in s["total"]]
    where = [s["table"][b].long()[slot // page] for b, slot in enumerate(slots)]

    def values(name, b):                          # [slots in use][kv_heads][d], and the exponents of their scales [slots in use][kv_heads]
        slot = slots[b]
        e = s[name + "_scales"][where[b], :, slot % page // block].to(wide) - 127
        return s[name].view(torch.uint8)[where[b], :, slot % page].view(torch.float8_e4m3fn).to(wide) * torch.exp2(e)[..., None], e

    if case["call"] == "append":                  # rows as they are before they are rounded, in units of their blocks' scales
        x = s["projected"].view(s["T"], H + 2 * Hk, d)
        turned = turn(x[:, :H + Hk], False)
        out, at = {"K": s["K"].to(wide), "V": s["V"].to(wide)}, 0
        for b in range(B):
            n, m = s["new_tokens"][b], s["total"][b]
            for name, rows in (("K", turned[at:at + n, H:]), ("V", x[at:at + n, H + Hk:].to(wide))):
                full, e = values(name, b)
                full[m - n:] = rows
                first = (m - n) // block * block  # the first slot whose block has new rows
                group = torch.arange(m - first, device="cuda") // block
                top = torch.zeros((int(group[-1]) + 1, Hk), device="cuda", dtype=wide).index_reduce_(0, group[m - n - first:], rows.abs().amax(-1), "amax")
                need = torch.ceil(torch.log2(top / 448.0)).clamp(_LEAST, _MOST)
                if first < m - n:
                    need[0] = torch.maximum(need[0], e[first])
                out[name][where[b][first:], :, slots[b][first:] % page] = full[first:] * torch.exp2(-need[group])[..., None]
            at += n
        return turned[:, :H], out["K"], None, out["V"], None
    at = 0
    O, lse = torch.zeros((s["T"], H, d), device="cuda", dtype=wide), torch.zeros((s["T"], H), device="cuda", dtype=wide)
    for b in range(B):
        n, length, slot = s["new_tokens"][b], s["total"][b], slots[b]
        query, first = slot[length - n:, None], min(case["prefix"], length)
        hidden = slot > query
        if case["window"]:
            hidden = hidden | (query - slot >= case["window"])
        hidden = hidden & (slot >= first)
        K, V = values("K", b)[0], values("V", b)[0]
        for h in range(H):
            z = s["Q"][at:at + n, h].to(wide) @ K[:, h // (H // Hk)].t().contiguous() / math.sqrt(d)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["slopes"]:
                z = z - s["slope"][h].to(wide) * (query - slot).abs()
            z = z.masked_fill(hidden, -math.inf)
            lse[at:at + n, h] = torch.logsumexp(z, 1)
            O[at:at + n, h] = torch.softmax(z, 1) @ V[:, h // (H // Hk)].contiguous()
        at += n
    return O, lse
