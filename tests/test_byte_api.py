"""Host-side checks of the paged cache in 8 bits and of rotary positions with several axes: what is refused, in which order, and how calls are marshalled."""
import inspect

import pytest

from paper_2407_13885_amd import binding
from test_api_cpu import BF16, E_ALIAS, E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_UNSUP, F32, OK
from test_paged_api import E_WORKSPACE, K, LENGTHS, LSE, O, Q, STARTS, TABLE, V, WORK, Lookalike, Number, _outcome, status

KS, VS = 0xa00000000, 0xb00000000


def cache(**more):
    at = dict(K=K, V=V, K_scales=KS, V_scales=VS, table=TABLE, lengths=LENGTHS, batch=2, pages=8, max_pages=4, page_size=16, block=8, kv_heads=2, d=64, dtype=BF16)
    at.update(more)
    return binding.AttnwByteCache(*at.values())


def attend(c=None, rule=None, q=Q, o=O, lse=LSE, starts=STARTS, tokens=3, heads=4, stride=256, work=WORK, size=1 << 30):
    return status("attnw_byte_paged_attention", c or cache(), rule or binding.AttnwRule(0.125), q, o, lse, starts, tokens, heads, stride, work, size)


def append(c=None, q=Q, k=Q + 0x1000, v=Q + 0x2000, r=O, table=WORK, positions=None, axes=None, starts=STARTS, tokens=3, heads=4, rot=64, rows=10, qs=256, kvs=128,
           layout=0):
    return status("attnw_byte_cache_append", c or cache(), q, k, v, r, table, positions, axes, starts, tokens, heads, rot, rows, qs, kvs, layout)


CACHES = [(dict(dtype=7), E_DTYPE), (dict(dtype=7, K=None), E_DTYPE), (dict(pages=-1), E_SHAPE), (dict(d=-64, K=None), E_SHAPE), (dict(block=-1), E_SHAPE),
          (dict(pages=1 << 40, page_size=1 << 40), E_SHAPE), (dict(K=None), E_NULL), (dict(V=None), E_NULL), (dict(table=None), E_NULL),
          (dict(lengths=None), E_NULL), (dict(K_scales=None), E_NULL), (dict(V_scales=None), E_NULL), (dict(d=24), E_UNSUP), (dict(d=272), E_UNSUP), (dict(d=0), E_UNSUP),
          (dict(d=36, dtype=F32), E_UNSUP), (dict(block=0), E_UNSUP), (dict(block=5), E_UNSUP), (dict(block=32), E_UNSUP), (dict(page_size=0), E_UNSUP),
          (dict(pages=0), E_UNSUP), (dict(max_pages=1 << 27), E_UNSUP), (dict(page_size=1 << 25), E_UNSUP), (dict(pages=1 << 30, page_size=1 << 16, block=1), E_UNSUP),
          (dict(K=K + 8), E_ALIGN), (dict(V=V + 2), E_ALIGN), (dict(table=TABLE + 2), E_ALIGN), (dict(lengths=LENGTHS + 1), E_ALIGN)]


@pytest.mark.parametrize("more,want", CACHES, ids=[str(c[0]) for c in CACHES])
def test_caches(more, want):
    d = max(0, more.get("d", 64))
    assert attend(cache(**more), stride=4 * d) == want
    assert append(cache(**more), rot=0, qs=4 * d, kvs=2 * d) == want


def test_attention():
    assert attend(cache(batch=0), q=None) == OK and attend(tokens=0, q=None) == OK and attend(heads=0, q=None) == OK
    for none in ("q", "o", "starts", "work"):
        assert attend(**{none: None}) == E_NULL, none
    assert attend(tokens=-1) == E_SHAPE and attend(heads=-4) == E_SHAPE and attend(stride=-1) == E_SHAPE and attend(size=-1) == E_SHAPE
    assert attend(rule=binding.AttnwRule(0.125, window=-1)) == E_SHAPE and attend(rule=binding.AttnwRule(0.125, cap=-2.0)) == E_SHAPE
    assert attend(rule=binding.AttnwRule(0.125, cap=float("nan"))) == E_SHAPE
    assert attend(rule=binding.AttnwRule(float("inf"))) == E_UNSUP and attend(rule=binding.AttnwRule(0.125, cap=float("inf"))) == E_UNSUP
    assert attend(heads=5, stride=320) == E_UNSUP and attend(stride=192) == E_UNSUP and attend(stride=260) == E_UNSUP
    assert attend(tokens=(1 << 30) + 1) == E_UNSUP and attend(tokens=1 << 45, stride=1 << 30) == E_SHAPE
    need = binding.attnw_byte_paged_workspace(cache(), 3, 4)
    assert need > 0 and attend(size=need - 1) == E_WORKSPACE
    for off in (dict(q=Q + 2), dict(o=O + 8), dict(lse=LSE + 2), dict(starts=STARTS + 1), dict(work=WORK + 4)):
        assert attend(**off) == E_ALIGN, off
    assert attend(rule=binding.AttnwRule(0.125, slopes=0x5002)) == E_ALIGN
    for both in (dict(o=Q), dict(o=K), dict(o=V + 4096), dict(lse=Q), dict(o=LSE), dict(lse=STARTS), dict(o=TABLE), dict(lse=LENGTHS), dict(o=KS), dict(lse=VS), dict(work=Q),
                 dict(work=O), dict(work=K), dict(work=VS)):
        assert attend(**both) == E_ALIAS, both
    assert binding.attnw_byte_paged_workspace(cache(batch=0), 3, 4) == 0
    for wrong in ((cache(), -1, 4), (cache(), 3, 5), (cache(block=3), 3, 4)):
        with pytest.raises(binding.AttnwError):
            binding.attnw_byte_paged_workspace(*wrong)
    assert status("attnw_byte_paged_attention", None, None, Q, O, LSE, STARTS, 3, 4, 256, WORK, 0) == E_NULL


def test_append():
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
    for both in (dict(k=K), dict(q=V), dict(r=K), dict(r=Q + 16), dict(r=WORK), dict(table=V + 64), dict(r=Q, qs=260), dict(k=KS), dict(r=VS), dict(r=TABLE), dict(r=LENGTHS)):
        assert append(**both) == E_ALIAS, both
    for more in (dict(K=TABLE), dict(V=LENGTHS), dict(K_scales=TABLE), dict(V_scales=KS), dict(V_scales=V + 64), dict(K_scales=K), dict(V=K), dict(table=VS + 4)):
        assert append(cache(**more)) == E_ALIAS, more
    axes = binding.AttnwAxes
    assert append(axes=axes([16, 16])) == E_NULL               # (no positions)
    assert append(axes=axes([16, 15]), positions=LSE) == E_UNSUP and append(axes=axes([32]), positions=LSE, rot=0) == E_UNSUP
    assert append(axes=axes([-1, 33]), positions=LSE) == E_SHAPE
    assert append(axes=axes([16, 16]), positions=O - 16, rows=10) == E_ALIAS   # two axes of three tokens: 24 bytes


def test_rotary_axes():
    axes = binding.AttnwAxes

    def rotary(x=Q, y=O, table=WORK, positions=STARTS, a=None, tokens=3, heads=4, d=64, rot=32, rows=10, xs=256, ys=256, layout=0, inverse=0, dtype=BF16):
        return status("attnw_rotary_axes", x, y, table, positions, a or axes([4, 6, 6]), tokens, heads, d, rot, rows, xs, ys, layout, inverse, dtype)
    assert rotary(dtype=3) == E_DTYPE and rotary(tokens=0, x=None) == OK and rotary(d=0, x=None) == OK
    for none in ("x", "y", "table", "positions"):
        assert rotary(**{none: None}) == E_NULL, none
    assert status("attnw_rotary_axes", Q, O, WORK, STARTS, None, 3, 4, 64, 32, 10, 256, 256, 0, 0, BF16) == E_NULL
    for wrong in (dict(rot=0), dict(rot=7), dict(rot=66), dict(rows=0), dict(layout=-1), dict(d=258, rot=2, xs=2000, ys=2000), dict(xs=255), dict(ys=1), dict(rot=30),
                  dict(a=axes([])), dict(a=axes([4, 4, 4, 3, 1])), dict(a=axes([4, 0, 12])), dict(a=axes([16], 2)), dict(a=axes([16], -1)), dict(a=axes([15])),
                  dict(a=axes([2 ** 31 - 1, 17]))):
        assert rotary(**wrong) == E_UNSUP, wrong
    assert rotary(heads=-1) == E_SHAPE and rotary(tokens=1 << 40, xs=1 << 40) == E_SHAPE and rotary(a=axes([17, -1])) == E_SHAPE
    assert rotary(x=Q + 2) == E_ALIGN and rotary(positions=STARTS + 2) == E_ALIGN
    assert rotary(y=Q, ys=260) == E_ALIAS and rotary(y=Q + 16) == E_ALIAS and rotary(y=WORK) == E_ALIAS and rotary(y=STARTS + 32) == E_ALIAS

    def table(table=Q, a=None, positions=4, rot=8, **more):
        return status_of_table(table, a or axes([1, 3]), positions, rot, **more)

    def status_of_table(*args, **more):
        try:
            binding.attnw_rotary_axes_table(*args, **more)
        except binding.AttnwError as e:
            return e.status
        return OK
    assert table(None, positions=0) == OK and table(None) == E_NULL and table(positions=-1) == E_SHAPE and table(Q + 4) == E_ALIGN
    for wrong in (dict(rot=10), dict(a=axes([2])), dict(base=0.0), dict(base=float("nan")), dict(factor=0.0), dict(low=3.0, high=2.0), dict(gain=float("inf")),
                  dict(original=-1.0)):
        assert table(**wrong) == E_UNSUP, wrong


def test_axes_take_numbers():
    with pytest.raises(TypeError):
        binding.AttnwAxes(["a"])
    assert list(binding.AttnwAxes((3, 4)).pairs) == [3, 4, 0, 0] and binding.AttnwAxes([1] * 7).count == 7


NAMES = ["attnw_rotary_axes", "attnw_byte_cache_append", "attnw_byte_paged_attention"]


@pytest.mark.parametrize("name", NAMES)
def test_the_callable_in_front_is_the_same_as_the_function(name):
    f = getattr(binding, name)
    plain = f.__wrapped__
    binding.load_library()
    assert f.__name__ == name and inspect.signature(f) == inspect.signature(plain) and binding._word_direct[name] is not None
    names = list(inspect.signature(plain).parameters)
    structures = dict(cache=cache(), rule=binding.AttnwRule(0.125), axes=binding.AttnwAxes([16, 16]))
    bad = []                                      # pointers off their alignment, numbers of nothing: whatever else there is, nothing is launched
    for n in names[:-1]:
        if n in structures:
            bad.append(structures[n])
        elif n in ("tokens", "heads", "d", "rot", "rows", "x_stride", "y_stride", "q_stride", "kv_stride", "layout", "inverse", "dtype", "workspace_bytes"):
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
    for wrong in (bad[:-1], bad + [None, None]):
        assert _outcome(f, wrong, {}) == _outcome(plain, wrong, {})


def test_structures_are_told_apart():
    """The cache of the other kind, another structure, or anything else that has an address, is refused by both ways in."""
    binding.load_library()
    rule, c, a = binding.AttnwRule(0.125), cache(), binding.AttnwAxes([16, 16])
    other = binding.AttnwCache(K, V, TABLE, LENGTHS, 2, 8, 4, 16, 2, 64, BF16)
    calls = dict(attnw_byte_cache_append=[c, Q, Q + 0x1000, Q + 0x2000, O, WORK, LSE, a, STARTS, 3, 4, 64, 10, 256, 128, 0],
                 attnw_byte_paged_attention=[c, rule, Q, O, LSE, STARTS, 3, 4, 256, WORK, 1 << 30],
                 attnw_rotary_axes=[Q, O, WORK, STARTS, a, 3, 4, 64, 64, 10, 256, 256, 0, 0, BF16])
    for name, right in calls.items():
        f = getattr(binding, name)
        for i, x in enumerate(right):
            if x is not c and x is not rule and x is not a:
                continue
            for wrong in (other, a if x is not a else c, Lookalike(), Lookalike, 7, "x"):
                for call in (f, f.__wrapped__):
                    with pytest.raises(TypeError, match="expected, not"):
                        call(*right[:i], wrong, *right[i + 1:])
    for wrong in (other, Lookalike()):
        with pytest.raises(TypeError, match="expected, not"):
            binding.attnw_byte_paged_workspace(wrong, 3, 4)
    with pytest.raises(TypeError, match="expected, not"):
        binding.attnw_paged_workspace(c, 3, 4)
