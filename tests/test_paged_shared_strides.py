"""Shared rows of caches whose rows lie apart: strides that attention without shared rows takes are taken with them too (no GPU here)."""
import ctypes as C

import pytest
import torch

from paper_2605_22269_amd import binding as mk
from test_paged_binding import SEQUENCES, Stand, tensors
from test_paged_refusals import BAD, UNSUP, pages, seqs


def size(p, bits=16):
    n = C.c_int64()
    rc = mk.load().mukv_paged_shared_workspace_size(C.byref(p), C.byref(seqs()), C.byref(seqs(n_seqs=2)), 0, C.byref(n))
    return rc, n.value


@pytest.mark.parametrize("dtype,row", [(mk.MUKV_BF16, 64 + 8), (mk.MUKV_F32, 64 + 4), (mk.MUKV_BF16, 64), (mk.MUKV_F32, 64 + 16)])
def test_rows_of_whole_pieces_are_taken(dtype, row):
    p = pages(dtype=dtype, stride_row=row, stride_head=row * 16, stride_page=row * 64, stride_layer=row * 6400)
    n = C.c_int64()
    assert mk.load().mukv_paged_workspace_size(C.byref(p), C.byref(seqs()), 0, C.byref(n)) == mk.MUKV_OK
    rc, m = size(p)
    assert rc == mk.MUKV_OK and m > n.value
    # bytes in 8 bits: no other space
    assert size(pages(dtype=dtype)) == size(p)


@pytest.mark.parametrize("kw,status", [({"stride_row": 66}, UNSUP), ({"stride_head": 2}, UNSUP), ({"stride_row": -64}, BAD), ({"stride_page": 1 << 60}, UNSUP)])
def test_others_are_refused(kw, status):
    assert size(pages(**kw))[0] == status
    assert size(pages(dtype=mk.MUKV_F32, **kw))[0] == status


@pytest.mark.parametrize("dtype,row", [(torch.bfloat16, 72), (torch.float32, 68)])
def test_the_python_call_takes_them(dtype, row, monkeypatch):
    at = lambda: Stand(1, 9, 2, 16, 64, dtype=dtype, strides=(row * 16 * 18, row * 32, row * 16, row, 1))  # noqa: E731
    c, reached = mk.PagedKV(at(), at(), n_q_heads=4), []
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: real(*a, **kw))
    monkeypatch.setattr(mk, "_stream_of", lambda index: 0)
    c._c_shared, c._c_capture = (lambda *a: reached.append(a[-2]) or 0), lambda stream, at: 0   # bytes of scratch
    kind = "b" if dtype is torch.bfloat16 else "f"
    t = tensors({}, **SEQUENCES, q=(kind, 3, 4, 64), out=(kind, 3, 4, 64))
    group = mk.Shared(*tensors({}, table=("i", 1, 6), lengths=("i", 1), offsets=("i", 2)).values())
    c.attend(0, **t, shared=group)
    assert len(reached) == 1 and reached[0] > 0
