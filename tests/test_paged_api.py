"""Host-side checks of the paged cache's entry points: what is refused, in which order, and how calls are marshalled."""
import inspect

import pytest

from paper_2407_13885_amd import binding
from test_api_cpu import BF16, E_ALIAS, E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_UNSUP, F32, OK

E_WORKSPACE = -8
K, V, TABLE, LENGTHS, Q, O, LSE, STARTS, WORK = (0x100000000 * (i + 1) for i in range(9))   # far apart: nothing is read


def cache(**more):
    at = dict(K=K, V=V, table=TABLE, lengths=LENGTHS, batch=2, pages=8, max_pages=4, page_size=16, kv_heads=2, d=64, dtype=BF16)
    at.update(more)
    return binding.AttnwCache(*(at[k] for k in ("K", "V", "table", "lengths", "batch", "pages", "max_pages", "page_size", "kv_heads", "d", "dtype")))


def status(name, *args):
    try:
        getattr(binding, name)(*args)
    except binding.AttnwError as e:
        return e.status
    return OK


def attend(c=None, rule=None, q=Q, o=O, lse=LSE, starts=STARTS, tokens=3, heads=4, stride=256, work=WORK, size=1 << 30):
    return status("attnw_paged_attention", c or cache(), rule or binding.AttnwRule(0.125), q, o, lse, starts, tokens, heads, stride, work, size)


CACHES = [(dict(dtype=7), E_DTYPE), (dict(dtype=7, K=None), E_DTYPE), (dict(pages=-1), E_SHAPE), (dict(d=-64, K=None), E_SHAPE),
          (dict(pages=1 << 40, page_size=1 << 40), E_SHAPE), (dict(K=None), E_NULL), (dict(V=None), E_NULL), (dict(table=None), E_NULL),
          (dict(lengths=None), E_NULL), (dict(d=24), E_UNSUP), (dict(d=272), E_UNSUP), (dict(d=0), E_UNSUP), (dict(d=6, dtype=F32), E_UNSUP),
          (dict(page_size=0), E_UNSUP), (dict(pages=0), E_UNSUP), (dict(max_pages=1 << 27), E_UNSUP), (dict(page_size=1 << 24), E_UNSUP), (dict(K=K + 8), E_ALIGN), (dict(V=V + 2), E_ALIGN),
          (dict(table=TABLE + 2), E_ALIGN), (dict(lengths=LENGTHS + 1), E_ALIGN)]


@pytest.mark.parametrize("more,want", CACHES, ids=[str(c[0]) for c in CACHES])
def test_caches(more, want):
    c = cache(**more)
    assert attend(c, heads=4, stride=4 * max(0, more.get("d", 64))) == want
    d = max(0, more.get("d", 64))
    assert status("attnw_cache_append", c, Q, Q + 0x1000, Q + 0x2000, O, WORK, None, STARTS, 3, 4, 0, 0, 4 * d, 2 * d, 0) == want
    if "V" not in more:                           # (sums do not look at V)
        assert status("attnw_paged_sums", c, binding.AttnwRule(0.125), Q, LSE, None, O, STARTS, 3, 4, 4 * d) == want
    if want != E_DTYPE:
        assert status("attnw_cache_evict", c, cache(K=Q, V=O, table=STARTS, lengths=WORK, **{k: v for k, v in more.items() if k in ("d", "dtype")}),
                      LSE, LSE + 0x100000, LSE + 0x200000, 8, 2) == want


def test_attention():
    assert attend(cache(batch=0), q=None) == OK and attend(tokens=0, q=None) == OK and attend(heads=0, q=None) == OK
    for none in ("q", "o", "starts", "work"):
        assert attend(**{none: None}) == E_NULL, none
    assert attend(tokens=-1) == E_SHAPE and attend(heads=-4) == E_SHAPE and attend(stride=-1) == E_SHAPE and attend(size=-1) == E_SHAPE
    assert attend(rule=binding.AttnwRule(0.125, window=-1)) == E_SHAPE and attend(rule=binding.AttnwRule(0.125, cap=-2.0)) == E_SHAPE
    assert attend(rule=binding.AttnwRule(0.125, cap=float("nan"))) == E_SHAPE
    assert attend(rule=binding.AttnwRule(float("inf"))) == E_UNSUP and attend(rule=binding.AttnwRule(0.125, cap=float("inf"))) == E_UNSUP
    assert attend(heads=5, stride=320) == E_UNSUP              # not a multiple of the kv heads
    assert attend(stride=192) == E_UNSUP and attend(stride=260) == E_UNSUP   # shorter than a row, not whole 16 bytes
    assert attend(tokens=(1 << 30) + 1) == E_UNSUP and attend(tokens=1 << 45, stride=1 << 30) == E_SHAPE
    need = binding.attnw_paged_workspace(cache(), 3, 4)
    assert need >= 0 and (need == 0 or attend(size=need - 1) == E_WORKSPACE)
    for off in (dict(q=Q + 2), dict(o=O + 8), dict(lse=LSE + 2), dict(starts=STARTS + 1), dict(work=WORK + 4)):
        assert attend(**off) == E_ALIGN, off
    assert attend(rule=binding.AttnwRule(0.125, slopes=0x5002)) == E_ALIGN
    for both in (dict(o=Q), dict(o=K), dict(o=V + 4096), dict(lse=Q), dict(o=LSE), dict(lse=STARTS), dict(o=TABLE), dict(lse=LENGTHS)):
        assert attend(**both) == E_ALIAS, both
    if need:
        assert attend(work=Q) == E_ALIAS and attend(work=O) == E_ALIAS and attend(work=K) == E_ALIAS
    assert binding.attnw_paged_workspace(cache(batch=0), 3, 4) == 0
    with pytest.raises(binding.AttnwError):
        binding.attnw_paged_workspace(cache(), -1, 4)
    with pytest.raises(binding.AttnwError):
        binding.attnw_paged_workspace(cache(), 3, 5)
    assert status("attnw_paged_attention", None, None, Q, O, LSE, STARTS, 3, 4, 256, WORK, 0) == E_NULL


def test_sums():
    def sums(c=None, q=Q, lse=LSE, before=None, out=O, starts=STARTS, tokens=3, heads=4, stride=256):
        return status("attnw_paged_sums", c or cache(), binding.AttnwRule(0.125), q, lse, before, out, starts, tokens, heads, stride)
    assert sums(cache(batch=0), q=None) == OK
    assert sums(q=None) == E_NULL and sums(lse=None) == E_NULL and sums(out=None) == E_NULL and sums(starts=None) == E_NULL
    assert sums(heads=0) == E_UNSUP and sums(heads=3) == E_UNSUP
    assert sums(out=O + 2) == E_ALIGN and sums(before=LSE + 1) == E_ALIGN
    assert sums(before=O + 4) == E_ALIAS and sums(out=K) == E_ALIAS and sums(out=LSE) == E_ALIAS


def test_append():
    def append(c=None, q=Q, k=Q + 0x1000, v=Q + 0x2000, r=O, table=WORK, positions=None, starts=STARTS, tokens=3, heads=4, rot=64, rows=10, qs=256, kvs=128,
               layout=0):
        return status("attnw_cache_append", c or cache(), q, k, v, r, table, positions, starts, tokens, heads, rot, rows, qs, kvs, layout)
    assert append(cache(batch=0), k=None) == OK and append(tokens=0, k=None) == OK
    for none in ("q", "k", "v", "r", "table", "starts"):
        assert append(**{none: None}) == E_NULL, none
    for wrong in (dict(rot=3), dict(rot=66), dict(rows=0), dict(layout=2), dict(qs=255), dict(kvs=127)):
        assert append(**wrong) == E_UNSUP, wrong
    assert append(tokens=-3) == E_SHAPE and append(rot=-2) == E_SHAPE
    for off in ("q", "k", "v", "r", "table"):
        at = dict(q=Q, k=Q + 0x1000, v=Q + 0x2000, r=O, table=WORK)[off]
        assert append(**{off: at + 4}) == E_ALIGN, off
    assert append(positions=LSE + 2) == E_ALIGN
    for both in (dict(k=K), dict(q=V), dict(r=K), dict(r=Q + 16), dict(r=WORK), dict(table=V + 64), dict(r=Q, qs=260)):
        assert append(**both) == E_ALIAS, both


def test_rotary():
    def rotary(x=Q, y=O, table=WORK, positions=STARTS, tokens=3, heads=4, d=64, rot=32, rows=10, xs=256, ys=256, layout=0, inverse=0, dtype=BF16):
        return status("attnw_rotary", x, y, table, positions, tokens, heads, d, rot, rows, xs, ys, layout, inverse, dtype)
    assert rotary(dtype=3) == E_DTYPE and rotary(tokens=0, x=None) == OK and rotary(d=0, x=None) == OK
    for none in ("x", "y", "table", "positions"):
        assert rotary(**{none: None}) == E_NULL, none
    for wrong in (dict(rot=0), dict(rot=7), dict(rot=66), dict(rows=0), dict(layout=-1), dict(d=258, rot=2, xs=2000, ys=2000), dict(xs=255), dict(ys=1)):
        assert rotary(**wrong) == E_UNSUP, wrong
    assert rotary(heads=-1) == E_SHAPE and rotary(tokens=1 << 40, xs=1 << 40) == E_SHAPE
    assert rotary(x=Q + 2) == E_ALIGN and rotary(positions=STARTS + 2) == E_ALIGN
    assert rotary(y=Q, ys=260) == E_ALIAS and rotary(y=Q + 16) == E_ALIAS and rotary(y=WORK) == E_ALIAS
    assert status("attnw_rotary_table", None, 0, 4) == OK and status("attnw_rotary_table", None, 4, 4) == E_NULL
    assert status("attnw_rotary_table", Q, -1, 4) == E_SHAPE and status("attnw_rotary_table", Q + 4, 4, 4) == E_ALIGN
    for wrong in (dict(rot=5), dict(rot=258), dict(base=0.0), dict(base=float("nan")), dict(factor=0.0), dict(low=3.0, high=2.0), dict(gain=float("inf")),
                  dict(original=-1.0)):
        at = dict(table=Q, positions=4, rot=4)
        at.update(wrong)
        with pytest.raises(binding.AttnwError) as e:
            binding.attnw_rotary_table(**at)
        assert e.value.status == E_UNSUP, wrong


def test_evict():
    def evict(c=None, into=None, sums=LSE, into_sums=LSE + 0x100000, kept=LSE + 0x200000, keep=8, recent=2):
        return status("attnw_cache_evict", c or cache(), into or cache(K=Q, V=O, table=STARTS, lengths=WORK), sums, into_sums, kept, keep, recent)
    away = dict(K=Q, V=O, table=STARTS, lengths=WORK)
    assert evict(cache(batch=0), cache(batch=0, **away)) == OK
    assert evict(sums=None) == E_NULL and evict(into_sums=None) == E_NULL and evict(kept=None) == E_NULL
    assert evict(into=cache(dtype=F32, **away)) == E_DTYPE and evict(into=cache(batch=3, **away)) == E_SHAPE and evict(into=cache(d=128, **away)) == E_SHAPE
    assert evict(keep=-1) == E_SHAPE and evict(recent=9) == E_SHAPE and evict(keep=0, recent=0) == E_UNSUP and evict(keep=65) == E_UNSUP
    assert evict(kept=LSE + 0x200002) == E_ALIGN
    assert evict(into=cache(**{**away, "K": V})) == E_ALIAS    # the new keys over the old values
    assert evict(into=cache(**{**away, "K": K + 16})) == E_ALIAS
    assert evict(into_sums=LSE) == E_ALIAS and evict(kept=LSE + 0x100000) == E_ALIAS and evict(into=cache(**{**away, "V": Q})) == E_ALIAS


NAMES = ["attnw_rotary", "attnw_cache_append", "attnw_paged_attention", "attnw_paged_sums", "attnw_cache_evict"]


def _outcome(f, args, kwargs):
    try:
        return f(*args, **kwargs)
    except Exception as e:                        # noqa: BLE001
        return type(e), str(e), getattr(e, "status", None)


class Number:
    def __index__(self):
        return 1


@pytest.mark.parametrize("name", NAMES)
def test_the_callable_in_front_is_the_same_as_the_function(name):
    f = getattr(binding, name)
    plain = f.__wrapped__
    binding.load_library()
    assert f.__name__ == name and inspect.signature(f) == inspect.signature(plain) and f.__globals__ is not None
    assert binding._word_direct[name] is not None
    names = list(inspect.signature(plain).parameters)
    c = cache()
    bad = []                                      # pointers off their alignment, numbers of nothing: whatever else there is, nothing is launched
    for n in names[:-1]:
        if n in ("cache", "into"):
            bad.append(c)
        elif n == "rule":
            bad.append(binding.AttnwRule(0.125))
        elif n in ("tokens", "heads", "d", "rot", "rows", "x_stride", "y_stride", "q_stride", "kv_stride", "layout", "inverse", "dtype", "workspace_bytes", "keep", "recent"):
            bad.append(-1)
        else:
            bad.append(Q + 1)
    for i in range(len(bad)):
        for v in (None, 0, -1, 1 << 40, 1 << 64, True, 1.5, "x", Number()):
            args = list(bad)
            args[i] = v
            assert _outcome(f, args, {}) == _outcome(plain, args, {}), (names[i], v)
    for stream in (None, 0, "x", 1 << 64):
        assert _outcome(f, bad + [stream], {}) == _outcome(plain, bad + [stream], {})
        assert _outcome(f, bad, {"stream": stream}) == _outcome(plain, bad, {"stream": stream})
    for wrong in (bad[:-1], bad + [None, None]):
        assert _outcome(f, wrong, {}) == _outcome(plain, wrong, {})


class Lookalike:
    _address = Q


def test_structures_are_told_apart():
    """One structure in the other's place, or anything else that has an address, is refused by both ways in: the host would read past its end."""
    binding.load_library()
    rule, c = binding.AttnwRule(0.125), cache()
    rest = dict(attnw_cache_append=[Q, Q + 0x1000, Q + 0x2000, O, WORK, None, STARTS, 3, 4, 64, 10, 256, 128, 0],
                attnw_paged_attention=[Q, O, LSE, STARTS, 3, 4, 256, WORK, 1 << 30], attnw_paged_sums=[Q, LSE, None, O, STARTS, 3, 4, 256],
                attnw_cache_evict=[LSE, LSE + 0x100000, LSE + 0x200000, 8, 2])
    for name, first in (("attnw_cache_append", [c]), ("attnw_paged_attention", [c, rule]), ("attnw_paged_sums", [c, rule]), ("attnw_cache_evict", [c, c])):
        f = getattr(binding, name)
        for i, right in enumerate(first):
            for wrong in (rule if right is c else c, Lookalike(), Lookalike, 7, "x"):
                args = first[:i] + [wrong] + first[i + 1:] + rest[name]
                for call in (f, f.__wrapped__):
                    with pytest.raises(TypeError, match="expected, not"):
                        call(*args)


def test_nothing_is_written_over_what_is_read():
    """Appending over the cache's own table and lengths, sums over its values."""
    def append(c=None, r=O):
        return status("attnw_cache_append", c or cache(), Q, Q + 0x1000, Q + 0x2000, r, WORK, None, STARTS, 3, 4, 64, 10, 256, 128, 0)

    def sums(out, **more):
        return status("attnw_paged_sums", cache(**more), binding.AttnwRule(0.125), Q, LSE, None, out, STARTS, 3, 4, 256)
    assert append(r=TABLE) == E_ALIAS and append(r=LENGTHS) == E_ALIAS
    for more in (dict(K=TABLE), dict(K=LENGTHS), dict(V=TABLE), dict(V=LENGTHS), dict(table=V + 64), dict(lengths=K + 1024)):
        assert append(cache(**more)) == E_ALIAS, more
    assert sums(V) == E_ALIAS and sums(V + 4096) == E_ALIAS
