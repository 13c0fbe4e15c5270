"""Eviction from a paged cache in 8 bits: rows and their scales move as they are.  Everything here is exact."""
import numpy as np
import pytest
import torch

from eight_testlib import random_cache, stands_for
from paged_testlib import spread_tables
from paper_2605_22269_amd import binding as mk
from test_gpu_paged_evict import BF16, F32, Case

pytestmark = pytest.mark.gpu


class Values:
    """What rows stand for, where Case asks for numbers of a tensor."""

    def __init__(self, pages, scales):
        self.parts = pages, scales

    detach = double = cpu = lambda self: self

    def numpy(self):
        return stands_for(*self.parts)


class Eight(Case):
    def __init__(self, lengths, R, D, hkv, layers, dtype, seed, order="page_head_row"):
        super().__init__(lengths, R, 16, hkv, layers, dtype, seed)
        kp, vp, ks, vs = random_cache(self.rng, (layers, self.n_pages, hkv, R, D), spread=20, order=order)
        self.cache = mk.PagedKV8(kp, vp, ks, vs, n_q_heads=hkv, dtype=dtype)
        self.kp, self.vp = Values(kp, ks), Values(vp, vs)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,D,order", [(BF16, 128, "page_head_row"), (F32, 64, "page_row_head"), (BF16, 16, "head_page_row"), (F32, 32, "page_head_row")])
@pytest.mark.parametrize("lengths,R,budget,sink,recent", [
    ([1], 1, 1, 0, 0), ([700], 16, 350, 4, 64), ([0, 5, 33, 900], 7, 33, 2, 8), ([64, 65, 2500], 64, 64, 0, 64), ([3000, 10], 24, 2999, 4, 0),
    ([513, 2049, 4097], 32, 500, 250, 250), ([40, 41], 8, 100, 3, 3)])
def test_eviction(lengths, R, budget, sink, recent, dtype, D, order, in_place):
    c = Eight(lengths, R, D, 2, 2, dtype, seed=sum(lengths) + R, order=order)
    c.check(budget, sink, recent, in_place=in_place, weights_in_place=in_place)


def test_rows_without_pages_are_never_kept():
    c = Eight([100, 90, 64], 16, 32, 2, 2, F32, seed=4)
    c.table[0, 2], c.table[0, 6] = -1, 2**31 - 1
    c.table[1, :] = -1
    c.into[2, 1] = c.n_pages
    c.check(50, 4, 20)
    c.check(95, 4, 20)


def test_again_and_again():
    c = Eight([300], 16, 128, 2, 2, BF16, seed=7)
    for _ in range(5):
        c.check(100, 4, 30, in_place=True, weights_in_place=False)
        c.w = c.rng.random(c.w.shape).astype(np.float32)
        c.lengths[:] = 120


def test_what_stays_is_attended_to_as_before():
    """Rows that nobody would miss: the outputs over what is left are those over a cache of these rows."""
    rng = np.random.default_rng(3)
    table, n_pages = spread_tables(rng, [200, 90], 16)
    kp, vp, ks, vs = random_cache(rng, (1, n_pages, 2, 16, 64))
    cache = mk.PagedKV8(kp, vp, ks, vs, n_q_heads=4)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    w = torch.rand(1, 2, 2, 200, device="cuda")
    k, v = stands_for(kp, ks)[0], stands_for(vp, vs)[0]
    kept, lengths = cache.evict(i32(table), i32([200, 90]), w, 50, sink=2, recent=8)
    off = i32([0, 50, 100])
    back = cache.read(0, i32(table), lengths, off, n_tokens=100)
    rows = kept[0].cpu().numpy()
    for b in range(2):
        for g in range(2):
            page, r = table[b][rows[b, g] // 16], rows[b, g] % 16
            for x, y in ((back[0], k), (back[1], v)):
                assert np.array_equal(x[50 * b:50 * b + 50, g].double().cpu().numpy(), y[page, g, r])
