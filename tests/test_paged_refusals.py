"""What the paged cache's calls refuse, on the host, before anything is launched (no GPU here: pointers are never followed)."""
import ctypes as C

import pytest

from paper_2605_22269_amd import binding as mk

P = 1 << 20  # stands for device memory


def pages(**kw):
    base = dict(k_pages=P, v_pages=P, stride_layer=4096 * 100, stride_page=4096, stride_head=1024, stride_row=64, n_layers=2, n_pages=100,
                page_rows=16, n_q_heads=8, n_kv_heads=4, head_dim=64, dtype=mk.MUKV_BF16, device_id=0)
    return mk.mukv_paged(**{**base, **kw})


def seqs(**kw):
    base = dict(table=P, lengths=P, offsets=P, n_seqs=3, table_width=10, n_tokens=5, max_new=0)
    return mk.mukv_seqs(**{**base, **kw})


def rope(**kw):
    return mk.mukv_rope_table(**{**dict(inv_freq=P, axis=P, n_rot=64, n_axes=3, pairing=0, inverse=0), **kw})


ST = mk.mukv_strides(0, 64, 64 * 16)
BAD, SHAPE, UNSUP = mk.MUKV_ERR_INVALID_ARG, mk.MUKV_ERR_SHAPE, mk.MUKV_ERR_UNSUPPORTED
PAGES = [({"k_pages": None}, BAD), ({"v_pages": None}, BAD), ({"n_layers": 0}, BAD), ({"n_pages": 0}, BAD), ({"page_rows": 0}, BAD),
         ({"n_kv_heads": 0}, BAD), ({"device_id": -1}, BAD), ({"dtype": 2}, BAD), ({"n_q_heads": 6}, SHAPE), ({"head_dim": 48}, UNSUP),
         ({"head_dim": 256}, UNSUP), ({"n_q_heads": 4 * 1025}, UNSUP), ({"stride_row": -64}, BAD), ({"stride_row": 68}, UNSUP),
         ({"stride_head": 4}, UNSUP), ({"stride_page": 1 << 60}, UNSUP), ({"k_pages": P + 8}, UNSUP), ({"page_rows": (1 << 24) + 1}, UNSUP)]
SEQS = [({"n_seqs": 0}, BAD), ({"n_seqs": 65537}, UNSUP), ({"table": None}, BAD), ({"lengths": None}, BAD), ({"table_width": 0}, BAD),
        ({"n_tokens": -1}, BAD), ({"max_new": -1}, BAD), ({"offsets": None}, SHAPE), ({"n_tokens": 1 << 29}, UNSUP),
        ({"table_width": 1 << 28}, UNSUP)]


def append(p=None, layer=0, s=None, k=P, ks=ST, v=P, vs=ST, q=P, qs=ST, qo=P, qos=ST, r=None, pos=P):
    ref = lambda x: None if x is None else C.byref(x)
    return mk.load().mukv_paged_append(ref(p or pages()), layer, ref(s or seqs()), k, ref(ks), v, ref(vs), q, ref(qs), qo, ref(qos), ref(r),
                                       pos, None)


@pytest.mark.parametrize("kw,status", PAGES)
def test_append_refuses_pages(kw, status):
    assert append(p=pages(**kw)) == status


@pytest.mark.parametrize("kw,status", SEQS)
def test_append_refuses_sequences(kw, status):
    assert append(s=seqs(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    ({"layer": -1}, BAD), ({"layer": 2}, BAD), ({"k": None}, BAD), ({"v": None}, BAD), ({"ks": None}, BAD), ({"q": None}, BAD),
    ({"qo": None}, BAD), ({"qs": None}, BAD), ({"k": P + 2}, UNSUP), ({"ks": mk.mukv_strides(0, 65, 1024)}, UNSUP),
    ({"vs": mk.mukv_strides(0, 64, -1024)}, BAD), ({"r": rope(), "pos": None}, BAD)])
def test_append_refuses_tensors(kw, status):
    assert append(**kw) == status


ROPES = [({"inv_freq": None}, BAD), ({"n_rot": 0}, BAD), ({"n_rot": 24}, UNSUP), ({"n_rot": 80}, SHAPE), ({"n_axes": 0}, BAD),
         ({"n_axes": 17}, BAD), ({"pairing": 2}, BAD), ({"inverse": 2}, BAD), ({"inv_freq": P + 4}, UNSUP)]


@pytest.mark.parametrize("kw,status", ROPES)
def test_rotations_are_refused_alike(kw, status):
    assert append(r=rope(**kw)) == status
    call = lambda r: mk.load().mukv_rope(C.byref(r), P, C.byref(ST), P, 4, 8, 64, mk.MUKV_BF16, P, C.byref(ST), 0, None)
    assert call(rope(**kw)) == status


@pytest.mark.parametrize("args,status", [
    (dict(T=-1), BAD), (dict(H=0), BAD), (dict(D=0), BAD), (dict(dtype=5), BAD), (dict(dev=-1), BAD), (dict(x=None), BAD), (dict(out=None), BAD),
    (dict(pos=None), BAD), (dict(D=68), UNSUP), (dict(D=1032), UNSUP), (dict(H=65536), UNSUP), (dict(x=P + 4), UNSUP)])
def test_rope_refuses(args, status):
    a = {**dict(T=4, H=8, D=64, dtype=mk.MUKV_BF16, dev=0, x=P, out=P, pos=P), **args}
    assert mk.load().mukv_rope(C.byref(rope()), a["x"], C.byref(ST), a["pos"], a["T"], a["H"], a["D"], a["dtype"], a["out"], C.byref(ST),
                               a["dev"], None) == status


def test_nothing_to_do_is_no_error():
    assert append(s=seqs(n_tokens=0)) == mk.MUKV_OK
    assert mk.load().mukv_rope(C.byref(rope()), P, C.byref(ST), P, 0, 8, 64, mk.MUKV_BF16, P, C.byref(ST), 0, None) == mk.MUKV_OK
    assert mk.load().mukv_paged_append(None, 0, C.byref(seqs()), P, None, P, None, None, None, None, None, None, None, None) == BAD
    assert mk.load().mukv_rope(None, P, C.byref(ST), P, 4, 8, 64, 0, P, C.byref(ST), 0, None) == BAD


# ---- attention ----
def attend(p=None, layer=0, s=None, q=P, qs=ST, causal=1, out=P, w=None, ws=P, n=1 << 40):
    ref = lambda x: None if x is None else C.byref(x)
    return mk.load().mukv_paged_attend(ref(p or pages()), layer, ref(s or seqs()), q, ref(qs), causal, out, ref(w), ws, n, None)


def weights(**kw):
    return mk.mukv_row_weights(**{**dict(in_=P, out=P, stride_layer=0, stride_seq=400, stride_head=100, rows=100, decay=1.0), **kw})


WEIGHTS = [({"out": None}, BAD), ({"rows": 0}, BAD), ({"stride_seq": -1}, BAD), ({"stride_head": -1}, BAD), ({"stride_layer": -1}, BAD),
           ({"decay": -0.5}, BAD), ({"decay": float("nan")}, BAD), ({"decay": float("inf")}, BAD), ({"out": P + 2}, UNSUP), ({"in_": P + 1}, UNSUP)]


@pytest.mark.parametrize("kw,status", PAGES)
def test_attend_refuses_pages(kw, status):
    assert attend(p=pages(**kw)) == status


@pytest.mark.parametrize("kw,status", [(k, s) for k, s in SEQS if k not in ({"table": None}, {"offsets": None})] + [
    ({"table": None, "offsets": None, "n_tokens": 6}, BAD), ({"offsets": None}, SHAPE)])
def test_attend_refuses_sequences(kw, status):
    assert attend(s=seqs(**kw)) == status


@pytest.mark.parametrize("kw,status", WEIGHTS)
def test_attend_refuses_weights(kw, status):
    assert attend(w=weights(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    ({"layer": -1}, BAD), ({"layer": 2}, BAD), ({"causal": 2}, BAD), ({"q": None}, BAD), ({"out": None}, BAD), ({"ws": None}, BAD),
    ({"n": 1000}, mk.MUKV_ERR_CAPACITY), ({"q": P + 8}, UNSUP), ({"out": P + 8}, UNSUP), ({"ws": P + 8}, UNSUP),
    ({"qs": mk.mukv_strides(0, 60, 1024)}, UNSUP), ({"qs": mk.mukv_strides(0, -64, 1024)}, BAD)])
def test_attend_refuses_tensors(kw, status):
    assert attend(**kw) == status


def test_workspace_size():
    call = lambda p, s, w, out: mk.load().mukv_paged_workspace_size(C.byref(p), C.byref(s), w, out)
    n, m = C.c_int64(), C.c_int64()
    assert call(pages(), seqs(), 0, C.byref(n)) == call(pages(), seqs(), 1, C.byref(m)) == mk.MUKV_OK
    assert m.value == n.value + 8 * 5 * 8 and n.value > 0
    assert call(pages(), seqs(), 2, C.byref(n)) == call(pages(), seqs(), 0, None) == BAD
    assert call(pages(n_pages=0), seqs(), 0, C.byref(n)) == BAD
    assert attend(s=seqs(n_tokens=0)) == mk.MUKV_OK


# ---- eviction ----
def evict(p=None, s=None, w=None, budget=50, sink=4, recent=10, into=P, width=5, kept=P, lengths=P):
    w = weights() if w is None else w
    return mk.load().mukv_paged_evict(C.byref(p or pages()), C.byref(s or seqs()), C.byref(w) if w else None, budget, sink, recent, into, width,
                                      kept, lengths, None)


@pytest.mark.parametrize("kw,status", PAGES)
def test_evict_refuses_pages(kw, status):
    assert evict(p=pages(**kw)) == status


@pytest.mark.parametrize("kw,status", [({"n_seqs": 0}, BAD), ({"table": None}, BAD), ({"lengths": None}, BAD), ({"table_width": 0}, BAD),
                                       ({"table_width": 1 << 28}, UNSUP)])
def test_evict_refuses_sequences(kw, status):
    assert evict(s=seqs(**kw)) == status


@pytest.mark.parametrize("kw,status", [x for x in WEIGHTS if "decay" not in x[0]] + [({"in_": None}, BAD)])
def test_evict_refuses_weights(kw, status):
    assert evict(w=weights(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    ({"budget": 0}, BAD), ({"sink": -1}, BAD), ({"recent": -1}, BAD), ({"sink": 41}, BAD), ({"width": 0}, BAD), ({"kept": None}, BAD),
    ({"lengths": None}, BAD), ({"w": 0}, BAD), ({"budget": (1 << 30) + 1}, UNSUP)])
def test_evict_refuses(kw, status):
    assert evict(**kw) == status


def test_stream_capture_refuses_no_place():
    assert mk.load().mukv_stream_capture(None, None) == BAD
