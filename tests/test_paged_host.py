"""What a call of the paged cache costs on the host before the C entry: where a launch takes a few microseconds, functions that are passed through on
the way count (a tenth of a microsecond each)."""
import sys

import pytest
import torch

from paper_2605_22269_amd import binding as mk
from test_paged_binding import Stand, i32


def entered(call):
    """Names of the functions of the binding that a call enters."""
    names = []

    def on(frame, event, arg):
        if event == "call" and frame.f_code.co_filename == mk.__file__:
            names.append(frame.f_code.co_name)

    sys.setprofile(on)
    try:
        call()
    finally:
        sys.setprofile(None)
    return names


@pytest.fixture
def cache(monkeypatch):
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: real(*a, **kw))
    monkeypatch.setattr(mk, "_raw_stream", lambda index: 0)
    c = mk.PagedKV(Stand(1, 9, 2, 16, 64), Stand(1, 9, 2, 16, 64), n_q_heads=4)
    c._c_attend = c._c_append = c._c_shared = lambda *a: 0
    c._c_capture = lambda stream, at: 0
    return c


def test_single_tokens_attention_goes_straight_to_the_library(cache):
    table, lengths, q, out = i32(3, 5), i32(3), Stand(3, 4, 64), Stand(3, 4, 64)
    call = lambda: cache.attend(0, table, lengths, q, out=out)  # noqa: E731
    call()                                                       # (scratch, strides)
    assert sorted(entered(call)) == ["_attend", "_sequences", "_stream_of", "attend"]


def test_shared_rows_add_their_own_structure(cache):
    table, lengths, q, out = i32(3, 5), i32(3), Stand(3, 4, 64), Stand(3, 4, 64)
    group = mk.Shared(i32(1, 6), i32(1), i32(2))
    call = lambda: cache.attend(0, table, lengths, q, out=out, shared=group)  # noqa: E731
    call()
    assert sorted(entered(call)) == ["_attend", "_sequences", "_stream_of", "attend", "pack"]
