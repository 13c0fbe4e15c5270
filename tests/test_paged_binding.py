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
    raised, was = [], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)

    def guarded(i):
        try:
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
