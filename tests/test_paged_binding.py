"""What the Python side of the paged cache hands to the C ABI (no GPU here: stand-ins for tensors, nothing is launched)."""
import ctypes as C
import sys
import threading

import pytest
import torch

from paper_2605_22269_amd import binding as mk


class Stand:
    """As much of a tensor on a device as the binding asks for; its address is its own and never followed."""

    at = 1 << 30

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, strides=None):
        Stand.at += 1 << 20
        self.shape, self.dtype, self._at, self._device = torch.Size(shape), dtype, Stand.at, device
        self._strides = tuple(strides or torch.empty(shape, device="meta").stride())

    device = property(lambda self: torch.device("cpu") if self._device < 0 else torch.device("cuda", self._device))
    is_cuda = property(lambda self: self._device >= 0)
    ndim = property(lambda self: len(self.shape))

    def get_device(self):
        return self._device

    def data_ptr(self):
        return self._at

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return self._strides == torch.empty(self.shape, device="meta").stride()


def threads(n, work):
    """n threads that change as often as they can; what they raised."""
    raised, was, together = [], sys.getswitchinterval(), threading.Barrier(n)
    sys.setswitchinterval(1e-6)

    def guarded(i):
        try:
            together.wait(60)   # (all of them are there: no number of a thread is given twice)
            work(i)
        except BaseException as e:  # noqa: BLE001
            raised.append(repr(e))

    try:
        all_of_them = [threading.Thread(target=guarded, args=(i,)) for i in range(n)]
        [t.start() for t in all_of_them]
        [t.join() for t in all_of_them]
    finally:
        sys.setswitchinterval(was)
    assert not raised, raised[:3]


def test_strides_of_several_threads_are_their_own():
    wrong = []

    def work(i):
        t = Stand(2, 2, 8)
        for n in range(20000):
            t._strides = (8 * (n * 8 + i) + 8, 8 * i, 1)
            got = mk.mukv_strides.from_buffer_copy(C.string_at(mk._rows(t), C.sizeof(mk.mukv_strides)))
            if (got.layer, got.head, got.token) != (0, t._strides[1], t._strides[0]):
                wrong.append((i, n))

    threads(8, work)
    assert not wrong, (len(wrong), wrong[:5])


def test_strides_are_not_kept_for_ever():
    for n in range(3000):
        mk._rows(Stand(2, 2, 8, strides=(16 * n, 8, 1)))
    assert len(mk._STRIDES) <= 1000


def test_strides_of_other_kinds_are_refused():
    for strides in ((16, 8, 2), (8, 1), (32, 16, 8, 1)):
        with pytest.raises(AssertionError):
            mk._rows(Stand(*[2] * len(strides), strides=strides))
    assert C.string_at(mk._rows(Stand(0, 2, 8, strides=(5, 5, 5))), 24) == bytes(24)


# ---- threads that use one cache ----
SLOW = 2e-5   # a call that takes its time before it reads what it was given


@pytest.fixture
def calls(monkeypatch):
    """What the C functions were given, read a while after the call: (thread, pages, seqs, weights, q or k)."""
    import time

    real, made = torch.empty, []
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: real(*a, **kw))   # (scratch, where there is no device)
    monkeypatch.setattr(mk, "_stream_of", lambda index: threading.get_ident())
    lib, held = mk.load(), []

    def stand_in(name, work):
        f = C.CFUNCTYPE(C.c_int, *getattr(lib, name).argtypes)(work)
        held.append(f)
        return f

    def read(kind, at):
        return kind.from_buffer_copy(C.string_at(at, C.sizeof(kind))) if at else None

    def append(pages, layer, s, k, *rest):
        time.sleep(SLOW)
        made.append((threading.get_ident(), read(mk.mukv_paged, pages), read(mk.mukv_seqs, s), None, k))
        return 0

    def attend(pages, layer, s, q, q_strides, causal, out, w, ws, ws_bytes, stream):
        time.sleep(SLOW)
        made.append((threading.get_ident(), read(mk.mukv_paged, pages), read(mk.mukv_seqs, s), read(mk.mukv_row_weights, w), q))
        assert stream == threading.get_ident()
        return 0

    def capture(stream, at):
        C.c_uint64.from_address(at).value = 0
        return 0

    def cache(c):
        c._c_append, c._c_attend = stand_in("mukv_paged_append", append), stand_in("mukv_paged_attend", attend)
        c._c_capture = stand_in("mukv_stream_capture", capture)
        return c

    yield cache, made


def i32(*shape):
    return Stand(*shape, dtype=torch.int32)


def test_threads_that_share_a_paged_cache_call_with_their_own_arguments(calls):
    cache, made = calls
    c = cache(mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4))
    given = {}

    def work(i):
        n, T = 2 + i, 5 * (2 + i)
        table, lengths, off = i32(n, 7 + i), i32(n), i32(n + 1)
        q, out, k, v = Stand(T, 4, 64), Stand(T, 4, 64), Stand(T, 2, 64), Stand(T, 2, 64)
        w, was = (Stand(n, 2, 50 + i, dtype=torch.float32) for _ in "ab")
        given[threading.get_ident()] = table, lengths, off, q, k, w, was, n, T
        for _ in range(100):
            c.append(0, table, lengths, k, v, offsets=off)
            c.attend(0, table, lengths, q, offsets=off, out=out, weights=was, weights_out=w, max_new=i)

    threads(6, work)
    assert len(made) == 1200
    for who, _, s, w_got, x in made:
        table, lengths, off, q, k, w, was, n, T = given[who]
        assert (s.table, s.lengths, s.offsets, s.n_seqs, s.table_width, s.n_tokens) == (
            table.data_ptr(), lengths.data_ptr(), off.data_ptr(), n, table.shape[1], T)
        assert x == (q if w_got else k).data_ptr()
        if w_got:
            assert (w_got.in_, w_got.out, w_got.rows) == (was.data_ptr(), w.data_ptr(), w.shape[2])


def test_threads_that_share_a_packed_cache_call_with_their_own_arguments(calls):
    cache, made = calls
    c = cache(mk.PackedKV(n_q_heads=4))
    given = {}

    def work(i):
        T, D, dt = 10 + i, (64, 128)[i % 2], (torch.bfloat16, torch.float32)[i // 2 % 2]
        q, out, k, v, off = Stand(T, 4, D, dtype=dt), Stand(T, 4, D, dtype=dt), Stand(T, 2, D, dtype=dt), Stand(T, 2, D, dtype=dt), i32(3 + i)
        given[threading.get_ident()] = q, k, v, off, T, D, mk.MUKV_BF16 if dt == torch.bfloat16 else mk.MUKV_F32
        for _ in range(200):
            c.attend(q, k, v, off, out=out)

    threads(6, work)
    assert len(made) == 1200
    for who, p, s, _, x in made:
        q, k, v, off, T, D, dt = given[who]
        assert (p.k_pages, p.v_pages, p.page_rows, p.head_dim, p.dtype, p.stride_row) == (k.data_ptr(), v.data_ptr(), T, D, dt, 2 * D)
        assert (s.offsets, s.n_seqs, s.n_tokens) == (off.data_ptr(), off.shape[0] - 1, T) and x == q.data_ptr()


def test_structures_are_packed_as_they_are_declared():
    for layout, kind in ((mk._SEQS, mk.mukv_seqs), (mk._WEIGHTS, mk.mukv_row_weights), (mk._PAGED, mk.mukv_paged)):
        assert layout.size == C.sizeof(kind)
        numbers = list(range(1, len(kind._fields_) + 1))
        got = kind.from_buffer_copy(layout.pack(*numbers))
        assert [getattr(got, name) for name, _ in kind._fields_] == numbers


# ---- tensors that lie elsewhere ----
PLACES = [-1, 1]   # host memory, another device


@pytest.fixture
def refuses(monkeypatch):
    """Nothing may be launched; a call with one of its tensors elsewhere raises."""
    reached = []
    for name in ("mukv_rope", "mukv_paged_append", "mukv_paged_attend", "mukv_paged_evict"):
        monkeypatch.setattr(mk, name, lambda *a: reached.append(a))
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: real(*a, **kw))
    monkeypatch.setattr(mk, "_stream_of", lambda index: 0)

    def check(call, names, place, cache=None):
        if cache is not None:
            cache._c_append = cache._c_attend = lambda *a: reached.append(a) or 0
            cache._c_capture = lambda stream, at: 0
        call({})
        assert reached, "the call itself goes through"
        reached.clear()
        for name in names:
            with pytest.raises(AssertionError):
                call({name: place})
            assert not reached, name

    return check


def tensors(where, **shapes):
    kinds = {"i": torch.int32, "f": torch.float32, "d": torch.float64, "b": torch.bfloat16}
    return {name: Stand(*shape, dtype=kinds[kind], device=where.get(name, 0)) for name, (kind, *shape) in shapes.items()}


@pytest.mark.parametrize("place", PLACES)
def test_rotations_refuse_tensors_that_lie_elsewhere(refuses, place):
    def call(where):
        t = tensors(where, inv_freq=("d", 16), axis=("i", 16), x=("b", 3, 2, 32), positions=("i", 2, 3), out=("b", 3, 2, 32))
        mk.Rope(t["inv_freq"], t["axis"], n_axes=2).rotate(t["x"], t["positions"], out=t["out"])

    refuses(call, ["inv_freq", "axis", "x", "positions", "out"], place)


SEQUENCES = dict(table=("i", 2, 5), lengths=("i", 2), offsets=("i", 3))


@pytest.mark.parametrize("place", PLACES)
def test_append_refuses_tensors_that_lie_elsewhere(refuses, place):
    c = mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4)

    def call(where):
        t = tensors(where, **SEQUENCES, k=("b", 3, 2, 64), v=("b", 3, 2, 64), q=("b", 3, 4, 64), q_out=("b", 3, 4, 64), positions=("i", 1, 3))
        rope = mk.Rope(Stand(16, dtype=torch.float64, device=max(where.get("rope", 0), 0)))
        c.append(0, **t, rope=rope)

    names = [*SEQUENCES, "k", "v", "q", "q_out", "positions"]
    refuses(call, names if place < 0 else [*names, "rope"], place, c)


@pytest.mark.parametrize("place", PLACES)
def test_attention_refuses_tensors_that_lie_elsewhere(refuses, place):
    c = mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4)
    rows = dict(q=("b", 3, 4, 64), out=("b", 3, 4, 64), weights=("f", 2, 2, 80), weights_out=("f", 2, 2, 80))
    refuses(lambda where: c.attend(0, **tensors(where, **SEQUENCES, **rows)), [*SEQUENCES, *rows], place, c)
    packed = mk.PackedKV(n_q_heads=4)
    rows = dict(rows, k=("b", 3, 2, 64), v=("b", 3, 2, 64), offsets=("i", 3))
    refuses(lambda where: packed.attend(**tensors(where, **rows)), rows, place, packed)


@pytest.mark.parametrize("place", PLACES)
def test_eviction_refuses_tensors_that_lie_elsewhere(refuses, place):
    c = mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4)
    rest = dict(table=("i", 2, 5), lengths=("i", 2), weights=("f", 1, 2, 2, 80), weights_out=("f", 1, 2, 2, 80), into=("i", 2, 5),
                kept=("i", 1, 2, 2, 40), lengths_out=("i", 2))
    refuses(lambda where: c.evict(budget=40, **tensors(where, **rest)), rest, place, c)


def test_pages_in_host_memory_are_refused():
    for where in ((-1, -1), (0, -1), (0, 1)):
        with pytest.raises(AssertionError):
            mk.PagedKV(*(Stand(1, 9, 2, 16, 64, device=d) for d in where), n_q_heads=4)
    with pytest.raises(AssertionError):   # real ones
        mk.PagedKV(torch.zeros(1, 2, 2, 4, 64), torch.zeros(1, 2, 2, 4, 64), n_q_heads=4)
    with pytest.raises(AssertionError):
        mk.Rope(torch.ones(16, dtype=torch.float64))


def test_packed_sequences_of_no_tokens_are_no_error(monkeypatch):
    """Empty tensors have no address; with weights or without, there is nothing to do."""
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: real(*a, **kw))
    monkeypatch.setattr(mk, "_stream_of", lambda index: 0)
    packed = mk.PackedKV(n_q_heads=4)
    packed._c_capture = lambda stream, at: 0
    t = dict(q=Stand(0, 4, 64), k=Stand(0, 2, 64), v=Stand(0, 2, 64), offsets=i32(3))
    for name in "qkv":
        t[name]._at = 0
    out, w = Stand(0, 4, 64), Stand(2, 2, 7, dtype=torch.float32)
    assert packed.attend(**t, out=out) is out and packed.attend(**t, out=out, weights_out=w) is out
    got = packed.attend(**t, weights=w, weights_out=w)
    assert got.shape == (0, 4, 64) and got is not t["q"] and packed.attend(**t) is not t["q"]


def test_packed_nothing_is_no_error_at_the_c_entry():
    pages = mk.mukv_paged(None, None, 0, 0, 64, 128, 1, 1, 0, 4, 2, 64, mk.MUKV_BF16, 0)
    seqs = mk.mukv_seqs(None, None, 1 << 20, 2, 0, 0, 0)
    rows = mk.mukv_row_weights(1 << 20, 1 << 20, 0, 14, 7, 7, 1.0)
    size = C.c_int64()
    lib, at = mk.load(), C.addressof
    assert lib.mukv_paged_workspace_size(at(pages), at(seqs), 1, C.byref(size)) == mk.MUKV_OK and size.value >= mk.MUKV_PAGED_CLEAR
    for w in (None, at(rows)):
        assert lib.mukv_paged_attend(at(pages), 0, at(seqs), None, None, 1, None, w, None, 0, None) == mk.MUKV_OK
    seqs.n_tokens = 3   # but of some tokens it is
    assert lib.mukv_paged_attend(at(pages), 0, at(seqs), 1 << 20, None, 1, 1 << 20, None, 1 << 20, 1 << 40, None) == mk.MUKV_ERR_INVALID_ARG
    seqs.n_tokens, seqs.table, seqs.lengths, seqs.table_width = 0, 1 << 20, 1 << 20, 4   # and of pages
    assert lib.mukv_paged_attend(at(pages), 0, at(seqs), None, None, 1, None, None, None, 0, None) == mk.MUKV_ERR_INVALID_ARG
