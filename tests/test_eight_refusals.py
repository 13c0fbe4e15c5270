"""What the calls on a cache in 8 bits refuse, on the host, before anything is launched (no GPU here: pointers are never followed)."""
import ctypes as C

import pytest
import torch

from paper_2605_22269_amd import binding as mk
from test_paged_binding import PLACES, SEQUENCES, Stand, refuses, tensors  # noqa: F401
from test_paged_refusals import BAD, P, SEQS, SHAPE, ST, UNSUP, WEIGHTS, pages, rope, seqs, weights

ref = lambda x: None if x is None else C.byref(x)  # noqa: E731


def scales(**kw):
    return mk.mukv_row_scales(**{**dict(k=P + 1, v=P + 3, stride_layer=6400, stride_page=64, stride_head=16, stride_row=1), **kw})


# strides of pages are bytes
PAGES8 = [({"k_pages": None}, BAD), ({"v_pages": None}, BAD), ({"n_layers": 0}, BAD), ({"n_pages": 0}, BAD), ({"page_rows": 0}, BAD),
          ({"n_kv_heads": 0}, BAD), ({"device_id": -1}, BAD), ({"dtype": 2}, BAD), ({"n_q_heads": 6}, SHAPE), ({"head_dim": 48}, UNSUP),
          ({"head_dim": 256}, UNSUP), ({"stride_row": -64}, BAD), ({"stride_row": 72}, UNSUP), ({"stride_head": 8}, UNSUP),
          ({"stride_page": 1 << 60}, UNSUP), ({"k_pages": P + 8}, UNSUP), ({"page_rows": (1 << 24) + 1}, UNSUP)]
SCALES = [(None, BAD), ({"k": None}, BAD), ({"v": None}, BAD), ({"stride_layer": -1}, BAD), ({"stride_page": -64}, BAD), ({"stride_head": -1}, BAD),
          ({"stride_row": -1}, BAD), ({"stride_page": 1 << 60}, UNSUP)]


def of(kw):
    return None if kw is None else scales(**kw)


def append(p=None, sc=scales(), layer=0, s=None, k=P, ks=ST, v=P, vs=ST, q=P, qs=ST, qo=P, qos=ST, r=None, pos=P):
    return mk.load().mukv_paged_append8(ref(p or pages()), ref(sc), layer, ref(s or seqs()), k, ref(ks), v, ref(vs), q, ref(qs), qo, ref(qos),
                                        ref(r), pos, None)


def read(p=None, sc=scales(), layer=0, s=None, k=P, ks=ST, v=P, vs=ST):
    return mk.load().mukv_paged_read8(ref(p or pages()), ref(sc), layer, ref(s or seqs()), k, ref(ks), v, ref(vs), None)


@pytest.mark.parametrize("call", [append, read])
def test_pages_scales_and_sequences_are_refused(call):
    for kw, status in PAGES8:
        assert call(p=pages(**kw)) == status, kw
    for kw, status in SCALES:
        assert call(sc=of(kw)) == status, kw
    for kw, status in SEQS:
        assert call(s=seqs(**kw)) == status, kw
    assert call(layer=-1) == call(layer=2) == BAD
    assert call(s=seqs(n_tokens=0)) == mk.MUKV_OK
    # a dimension of one is never walked
    one = dict(n_layers=1, stride_layer=-5)
    assert call(p=pages(**one), sc=scales(stride_layer=-5), s=seqs(n_tokens=0)) == mk.MUKV_OK


@pytest.mark.parametrize("kw,status", [
    ({"k": None}, BAD), ({"v": None}, BAD), ({"ks": None}, BAD), ({"q": None}, BAD), ({"qo": None}, BAD), ({"qs": None}, BAD),
    ({"k": P + 2}, UNSUP), ({"ks": mk.mukv_strides(0, 65, 1024)}, UNSUP), ({"vs": mk.mukv_strides(0, 64, -1024)}, BAD),
    ({"r": rope(), "pos": None}, BAD), ({"r": rope(n_rot=24)}, UNSUP), ({"r": rope(n_rot=80)}, SHAPE)])
def test_append_refuses_tensors(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [({"k": None}, BAD), ({"v": None}, BAD), ({"ks": None}, BAD), ({"vs": None}, BAD), ({"v": P + 2}, UNSUP),
                                       ({"ks": mk.mukv_strides(0, 65, 1024)}, UNSUP), ({"vs": mk.mukv_strides(0, 64, -1024)}, BAD)])
def test_read_refuses_tensors(kw, status):
    assert read(**kw) == status


# ---- the Python side ----
def cache8(where={}, dtype=torch.bfloat16, **kw):
    e, s = torch.float8_e4m3fn, torch.float8_e8m0fnu
    at = lambda name, *shape, dtype: Stand(*shape, dtype=dtype, device=where.get(name, 0), **kw.get(name, {}))  # noqa: E731
    return mk.PagedKV8(at("k_pages", 1, 9, 2, 16, 64, dtype=e), at("v_pages", 1, 9, 2, 16, 64, dtype=e), at("k_scales", 1, 9, 2, 16, dtype=s),
                       at("v_scales", 1, 9, 2, 16, dtype=s), n_q_heads=4, dtype=dtype)


@pytest.mark.parametrize("place", PLACES)
def test_caches_whose_parts_lie_apart_are_refused(place):
    cache8()
    for name in ("k_pages", "v_pages", "k_scales", "v_scales"):
        with pytest.raises(AssertionError):
            cache8({name: place})


def test_caches_of_other_types_and_shapes_are_refused():
    e, s = torch.float8_e4m3fn, torch.float8_e8m0fnu
    good = dict(k_pages=Stand(1, 9, 2, 16, 64, dtype=e), v_pages=Stand(1, 9, 2, 16, 64, dtype=e), k_scales=Stand(1, 9, 2, 16, dtype=s),
                v_scales=Stand(1, 9, 2, 16, dtype=s))
    mk.PagedKV8(**good, n_q_heads=4)
    for name, other in (("k_pages", Stand(1, 9, 2, 16, 64)), ("v_pages", Stand(1, 9, 2, 16, 64, dtype=torch.float8_e5m2)),
                        ("k_scales", Stand(1, 9, 2, 16, dtype=torch.float32)), ("v_scales", Stand(1, 9, 2, 16, dtype=torch.uint8)),
                        ("v_scales", Stand(1, 9, 2, 15, dtype=s)), ("v_scales", Stand(1, 9, 2, 16, dtype=s, strides=(0, 16, 144, 1))),
                        ("v_pages", Stand(1, 9, 2, 16, 32, dtype=e))):
        with pytest.raises(AssertionError):
            mk.PagedKV8(**{**good, name: other}, n_q_heads=4)
    with pytest.raises(AssertionError):
        mk.PagedKV8(**good, n_q_heads=4, dtype=torch.float16)


@pytest.mark.parametrize("place", PLACES)
def test_tensors_that_lie_elsewhere_are_refused(refuses, place, monkeypatch):  # noqa: F811
    c = cache8()
    kv = dict(k=("b", 3, 2, 64), v=("b", 3, 2, 64))

    def put(where):
        t = tensors(where, **SEQUENCES, **kv, q=("b", 3, 4, 64), q_out=("b", 3, 4, 64), positions=("i", 1, 3))
        c.append(0, **t, rope=mk.Rope(Stand(16, dtype=torch.float64)))

    refuses(put, [*SEQUENCES, *kv, "q", "q_out", "positions"], place, c)
    reached = []
    monkeypatch.setattr(mk, "mukv_paged_read8", lambda *a: reached.append(a))

    def back(where):
        c.read(0, **tensors(where, **SEQUENCES, k_out=("b", 3, 2, 64), v_out=("b", 3, 2, 64)))

    back({})
    assert reached
    for name in (*SEQUENCES, "k_out", "v_out"):
        with pytest.raises(AssertionError):
            back({name: place})
    assert len(reached) == 1
    for kw in (dict(n_tokens=4, k_out=Stand(3, 2, 64)), dict(k_out=Stand(3, 2, 64), v_out=Stand(3, 2, 32)), dict(k_out=Stand(3, 2, 64, dtype=torch.float32))):
        with pytest.raises(AssertionError):
            c.read(0, **tensors({}, **SEQUENCES), **kw)


def test_structures_are_declared_as_they_are():
    assert C.sizeof(mk.mukv_row_scales) == 48
    c = cache8()
    assert (c._scales.k, c._scales.stride_page, c._scales.stride_head, c._scales.stride_row) == (c._held[2].data_ptr(), 32, 16, 1)
    assert (c._pages.stride_row, c._pages.dtype) == (64, mk.MUKV_BF16) and cache8(dtype=torch.float32)._pages.dtype == mk.MUKV_F32


# ---- attention ----
def attend(p=None, sc=scales(), layer=0, s=None, q=P, qs=ST, causal=1, out=P, w=None, ws=P, n=1 << 40):
    return mk.load().mukv_paged_attend8(ref(p or pages()), ref(sc), layer, ref(s or seqs()), q, ref(qs), causal, out, ref(w), ws, n, None)


GROUPS = dict(n_seqs=2, n_tokens=5)


def shared(p=None, sc=scales(), layer=0, s=None, g=seqs(**GROUPS), q=P, qs=ST, causal=1, out=P, w=None, sw=None, ws=P, n=1 << 40):
    return mk.load().mukv_paged_attend_shared(ref(p or pages()), ref(sc), layer, ref(s or seqs()), ref(g), q, ref(qs), causal, out, ref(w), ref(sw),
                                              ws, n, None)


@pytest.mark.parametrize("call", [attend, shared])
def test_attention_refuses_pages_scales_and_sequences(call):
    for kw, status in PAGES8:
        assert call(p=pages(**kw)) == status, kw
    for kw, status in SCALES:
        if call is attend or kw is not None:      # (without scales the rows are of the payload dtype)
            assert call(sc=of(kw)) == status, kw
    for kw, status in SEQS:
        if "offsets" not in kw:
            assert call(s=seqs(**kw)) == status, kw
    assert call(s=seqs(offsets=None)) == SHAPE and call(s=seqs(table=None, lengths=None)) == BAD
    assert call(layer=-1) == call(layer=2) == call(causal=2) == BAD


@pytest.mark.parametrize("call", [attend, shared])
@pytest.mark.parametrize("kw,status", [
    ({"q": None}, BAD), ({"out": None}, BAD), ({"ws": None}, BAD), ({"n": 1000}, mk.MUKV_ERR_CAPACITY), ({"q": P + 8}, UNSUP), ({"out": P + 8}, UNSUP),
    ({"ws": P + 8}, UNSUP), ({"qs": mk.mukv_strides(0, 60, 1024)}, UNSUP), ({"qs": mk.mukv_strides(0, -64, 1024)}, BAD)])
def test_attention_refuses_tensors(call, kw, status):
    assert call(**kw) == status


def test_attention_refuses_weights_and_groups():
    for kw, status in WEIGHTS:
        assert attend(w=weights(**kw)) == shared(w=weights(**kw)) == shared(sw=weights(**kw)) == status, kw
    assert shared(g=None) == BAD
    for kw, status in SEQS:
        if "offsets" not in kw:
            assert shared(g=seqs(**{**GROUPS, **kw})) == status, kw
    assert shared(g=seqs(n_seqs=2, offsets=None)) == SHAPE        # 5 tokens are not 2 groups of as many
    assert shared(g=seqs(n_tokens=4)) == SHAPE                    # not the call's tokens
    assert attend(s=seqs(n_tokens=0)) == shared(s=seqs(n_tokens=0), g=seqs(n_tokens=0)) == mk.MUKV_OK
    # pages of the payload dtype: strides are its elements
    assert shared(sc=None, p=pages(stride_row=68)) == UNSUP and shared(sc=None, s=seqs(n_tokens=0), g=seqs(n_tokens=0)) == mk.MUKV_OK


def test_shared_workspace_size():
    call = lambda p, s, g, w, out: mk.load().mukv_paged_shared_workspace_size(ref(p), ref(s), ref(g), w, out)  # noqa: E731
    plain, n, m = C.c_int64(), C.c_int64(), C.c_int64()
    assert mk.load().mukv_paged_workspace_size(ref(pages()), ref(seqs()), 0, C.byref(plain)) == mk.MUKV_OK
    assert call(pages(), seqs(), seqs(**GROUPS), 0, C.byref(n)) == call(pages(), seqs(), seqs(**GROUPS), 1, C.byref(m)) == mk.MUKV_OK
    assert n.value >= plain.value + 5 * 8 * (4 * 64 + 16) and m.value >= n.value + 8 * 5 * 8
    assert call(pages(), seqs(), None, 0, C.byref(n)) == call(pages(), None, seqs(), 0, C.byref(n)) == call(None, seqs(), seqs(), 0, C.byref(n)) == BAD
    assert call(pages(), seqs(), seqs(), 2, C.byref(n)) == call(pages(), seqs(), seqs(), 0, None) == BAD
    assert call(pages(), seqs(), seqs(n_tokens=3), 0, C.byref(n)) == SHAPE
    # rows that may be many chunks: a place for the queries of each
    wide = pages(head_dim=128, n_q_heads=32)
    one = seqs(n_seqs=64, n_tokens=64, offsets=None, max_new=1)
    assert call(wide, one, seqs(n_seqs=1, n_tokens=64, max_new=64, table_width=1), 0, C.byref(n)) == mk.MUKV_OK
    assert call(wide, one, seqs(n_seqs=1, n_tokens=64, max_new=64, table_width=40000), 0, C.byref(m)) == mk.MUKV_OK
    assert m.value > n.value + 100 * 128 * (4 * 128 + 16)


@pytest.mark.parametrize("place", PLACES)
def test_attention_refuses_tensors_that_lie_elsewhere(refuses, place):  # noqa: F811
    c = cache8()
    rows = dict(q=("b", 3, 4, 64), out=("b", 3, 4, 64), weights=("f", 2, 2, 80), weights_out=("f", 2, 2, 80))
    refuses(lambda where: c.attend(0, **tensors(where, **SEQUENCES, **rows)), [*SEQUENCES, *rows], place, c)
    for c in (cache8(), mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4)):
        reached = []
        c._c_shared, c._c_capture = (lambda *a: reached.append(a) or 0), lambda stream, at: 0
        more = dict(rows, shared_weights=("f", 1, 2, 90), shared_weights_out=("f", 1, 2, 90))
        group = {f"of_{k}": v for k, v in dict(table=("i", 1, 6), lengths=("i", 1), offsets=("i", 2)).items()}

        def call(where):
            t = tensors(where, **SEQUENCES, **more, **group)
            s = mk.Shared(*(t.pop(k) for k in group))
            c.attend(0, **t, shared=s)

        call({})
        assert len(reached) == 1 and (reached[0][1] is None) == (not isinstance(c, mk.PagedKV8))
        for name in (*SEQUENCES, *more, *group):
            with pytest.raises(AssertionError):
                call({name: place})
        assert len(reached) == 1
        with pytest.raises(AssertionError):      # nothing is shared
            t = tensors({}, **SEQUENCES, **more)
            c.attend(0, **t)
        with pytest.raises(AssertionError):      # all of it elsewhere
            mk_shared = mk.Shared(*tensors({f"of_{k}": 1 for k in ("table", "lengths", "offsets")}, **group).values())
            c.attend(0, **tensors({}, **SEQUENCES, **rows), shared=mk_shared)


def test_groups_are_packed_as_they_are_declared():
    t = tensors({}, table=("i", 3, 7), lengths=("i", 3), offsets=("i", 4))
    s = mk.mukv_seqs.from_buffer_copy(mk.Shared(*t.values(), max_tokens=9).pack(11))
    assert (s.table, s.lengths, s.offsets) == tuple(x.data_ptr() for x in t.values())
    assert (s.n_seqs, s.table_width, s.n_tokens, s.max_new) == (3, 7, 11, 9)
    assert mk.mukv_seqs.from_buffer_copy(mk.Shared(t["table"], t["lengths"]).pack(6)).offsets is None
    for bad in (dict(lengths=Stand(2, dtype=torch.int32)), dict(offsets=Stand(3, dtype=torch.int32)), dict(table=Stand(3, 7, dtype=torch.int64)),
                dict(table=Stand(3, 7, dtype=torch.int32, strides=(8, 1)))):
        with pytest.raises(AssertionError):
            mk.Shared(*{**t, **bad}.values())


# ---- eviction ----
def evict(p=None, sc=scales(), s=None, w=None, budget=50, sink=4, recent=10, into=P, width=5, kept=P, lengths=P):
    w = weights() if w is None else w
    return mk.load().mukv_paged_evict8(ref(p or pages()), ref(sc), ref(s or seqs()), ref(w) if w else None, budget, sink, recent, into, width, kept,
                                       lengths, None)


def test_evict_refuses():
    for kw, status in PAGES8:
        assert evict(p=pages(**kw)) == status, kw
    for kw, status in SCALES:
        assert evict(sc=of(kw)) == status, kw
    for kw, status in [x for x in WEIGHTS if "decay" not in x[0]] + [({"in_": None}, BAD)]:
        assert evict(w=weights(**kw)) == status, kw
    for kw, status in [({"n_seqs": 0}, BAD), ({"table": None}, BAD), ({"lengths": None}, BAD), ({"table_width": 0}, BAD), ({"table_width": 1 << 28}, UNSUP)]:
        assert evict(s=seqs(**kw)) == status, kw
    for kw, status in [({"budget": 0}, BAD), ({"sink": -1}, BAD), ({"recent": -1}, BAD), ({"sink": 41}, BAD), ({"width": 0}, BAD), ({"kept": None}, BAD),
                       ({"lengths": None}, BAD), ({"w": 0}, BAD), ({"budget": (1 << 30) + 1}, UNSUP)]:
        assert evict(**kw) == status, kw


@pytest.mark.parametrize("place", PLACES)
def test_eviction_refuses_tensors_that_lie_elsewhere(place, monkeypatch):
    c, reached = cache8(), []
    monkeypatch.setattr(mk, "mukv_paged_evict8", lambda *a: reached.append(a))
    monkeypatch.setattr(mk, "mukv_paged_evict", lambda *a: pytest.fail("rows of 16 bits"))
    monkeypatch.setattr(mk, "_stream_of", lambda index: 0)
    rest = dict(table=("i", 2, 5), lengths=("i", 2), weights=("f", 1, 2, 2, 80), weights_out=("f", 1, 2, 2, 80), into=("i", 2, 5),
                kept=("i", 1, 2, 2, 40), lengths_out=("i", 2))
    c.evict(budget=40, **tensors({}, **rest))
    assert len(reached) == 1 and reached[0][1] == c._scales_at
    for name in rest:
        with pytest.raises(AssertionError):
            c.evict(budget=40, **tensors({name: place}, **rest))
    assert len(reached) == 1
