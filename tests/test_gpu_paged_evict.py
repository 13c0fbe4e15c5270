"""Eviction from a paged cache: which rows stay, and where their keys, values and weights go.  Everything here is exact."""
import numpy as np
import pytest
import torch

from paged_testlib import f64, on_device, places, spread_tables
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def chosen(w, there, n, budget, sink, recent):
    """Rows that stay of one list, ascending: w [n] (NaN below all), there [n]."""
    j = np.arange(n)
    always = (j < sink) | (j >= n - recent)
    w = w.astype(np.float64)
    key = np.where(np.isnan(w), -2.0, np.where(np.isneginf(w), -1.0, 0.0))   # NaN, then -inf, then the numbers
    order = sorted(j[there], key=lambda i: (not always[i], -key[i], -w[i] if np.isfinite(w[i]) or w[i] == np.inf else 0.0, i))
    return np.sort(np.array(order[:budget], int))


class Case:
    def __init__(self, lengths, R, D, hkv, layers, dtype, seed, order="page_head_row", rows=None, ties=0.3):
        rng = self.rng = np.random.default_rng(seed)
        self.lengths, self.R, self.hkv, self.L, self.dtype = np.array(lengths, np.int32), R, hkv, layers, dtype
        self.table, used = spread_tables(rng, lengths, R, n_spare=0)
        self.into, fresh = spread_tables(rng, lengths, R, n_spare=2)
        self.into = np.where(self.into >= 0, self.into + used, -1).astype(np.int32)
        self.n_pages = used + fresh
        shape = (layers, self.n_pages, hkv, R, D)
        self.kp, self.vp = (on_device(rng.standard_normal(shape).astype(np.float32), dtype, order) for _ in "kv")
        N = rows or max(max(lengths), 1) + 3
        w = np.exp(2 * rng.standard_normal((layers, len(lengths), hkv, N))).astype(np.float32)
        self.w = np.where(rng.random(w.shape) < ties, rng.integers(0, 2, w.shape).astype(np.float32), w)
        self.cache = mk.PagedKV(self.kp, self.vp, n_q_heads=hkv)

    def check(self, budget, sink=0, recent=0, in_place=False, weights_in_place=False):
        k0, v0 = f64(self.kp), f64(self.vp)
        table, lengths = torch.tensor(self.table, device="cuda"), torch.tensor(self.lengths, device="cuda")
        into_t = None if in_place else torch.tensor(self.into, device="cuda")
        w = torch.tensor(self.w, device="cuda")
        w_out = w if weights_in_place else torch.full_like(w, 6.0)
        kept, after = self.cache.evict(table, lengths, w, budget, sink=sink, recent=recent, into=into_t, weights_out=w_out,
                                       lengths_out=lengths if in_place else None)
        want_k, want_v, into = k0.copy(), v0.copy(), self.table if in_place else self.into
        kept, w_out = kept.cpu().numpy(), w_out.cpu().numpy()
        room = self.table.shape[1] * self.R
        for b in range(len(self.lengths)):
            n = min(max(int(self.lengths[b]), 0), room)
            page, r, there = places(self.table, self.lengths, self.R, self.n_pages, b, np.arange(n))
            m = min(budget, int(there.sum()))
            assert after[b] == m
            for layer in range(self.L):
                for g in range(self.hkv):
                    wl = np.zeros(n, np.float32)
                    have = min(n, self.w.shape[3])
                    wl[:have] = self.w[layer, b, g, :have]
                    stay = chosen(wl, there, n, budget, sink, recent)
                    assert np.array_equal(kept[layer, b, g, :m], stay) and (kept[layer, b, g, m:] == -1).all()
                    to, tr, ok = places(into, self.lengths, self.R, self.n_pages, b, np.arange(m))
                    for x, y in ((want_k, k0), (want_v, v0)):
                        x[layer, to[ok], g, tr[ok]] = y[layer, page[stay][ok], g, r[stay][ok]]
                    expect = (self.w if weights_in_place else np.full_like(self.w, 6.0))[layer, b, g].copy()
                    expect[min(m, have):have] = 0.0
                    expect[: min(m, have)] = wl[stay][: min(m, have)]
                    assert np.array_equal(w_out[layer, b, g], expect, equal_nan=True)
        assert np.array_equal(f64(self.kp), want_k) and np.array_equal(f64(self.vp), want_v)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,D,order", [(BF16, 128, "page_head_row"), (F32, 64, "page_row_head"), (BF16, 16, "head_page_row"), (F32, 128, "page_head_row")])
@pytest.mark.parametrize("lengths,R,budget,sink,recent", [
    ([1], 1, 1, 0, 0), ([700], 16, 350, 4, 64), ([0, 5, 33, 900], 7, 33, 2, 8), ([64, 65, 2500], 64, 64, 0, 64), ([3000, 10], 24, 2999, 4, 0),
    ([513, 2049, 4097], 32, 500, 250, 250), ([40, 41], 8, 100, 3, 3)])
def test_eviction(lengths, R, budget, sink, recent, dtype, D, order, in_place):
    c = Case(lengths, R, D, 2, 2, dtype, seed=sum(lengths) + R, order=order)
    c.check(budget, sink, recent, in_place=in_place, weights_in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_more_rows_than_keys_wait_in_lds(in_place):
    c = Case([50003, 33000], 16, 16, 1, 1, BF16, seed=1)
    c.check(20000, 4, 100, in_place=in_place, weights_in_place=in_place)


@pytest.mark.parametrize("weights", ["equal", "few values", "no numbers", "small"])
def test_weights_that_tie_or_are_no_numbers(weights):
    c = Case([1000, 77], 16, 32, 2, 1, BF16, seed=2)
    if weights == "equal":
        c.w[:] = 0.25
    elif weights == "few values":
        c.w = c.rng.choice(np.array([0.0, -0.0, 1.0, 1e-30, 2.0], np.float32), c.w.shape)
    elif weights == "small":   # neighbours in the last bit, denormal numbers among them
        c.w = (c.rng.integers(0, 300, c.w.shape)).astype(np.uint32).view(np.float32)
    else:
        c.w = c.rng.choice(np.array([np.nan, np.inf, -np.inf, 1.0, -1.0], np.float32), c.w.shape)
    for budget in (1, 60, 400, 999):
        c.check(budget, sink=min(1, budget - 1))


def test_rows_without_pages_are_never_kept():
    c = Case([100, 90, 64], 16, 32, 2, 2, F32, seed=4)
    c.table[0, 2], c.table[0, 6] = -1, 2**31 - 1
    c.table[1, :] = -1
    c.into[2, 1] = c.n_pages      # rows that go there are lost
    c.check(50, 4, 20)
    c.check(95, 4, 20)
    c = Case([100, 90, 64], 16, 32, 2, 2, F32, seed=5)
    c.table[0, 0], c.table[1, 3] = -1, -(2**31)
    c.into[:] = -1
    c.check(80, 4, 20)


def test_lengths_past_the_table_and_fewer_weights_than_rows():
    c = Case([64, 200, 16], 16, 32, 1, 1, BF16, seed=6, rows=120)
    c.lengths[:] = [2**31 - 1, 200, -5]
    c.check(90, 4, 30)
    c = Case([64, 200, 16], 16, 32, 1, 1, BF16, seed=6, rows=120)
    c.check(150, 4, 30, in_place=True, weights_in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
def test_many_lists(in_place):
    rng = np.random.default_rng(9)
    c = Case([int(x) for x in rng.integers(0, 700, 40)], 16, 16, 4, 2, BF16, seed=10)
    c.check(200, 4, 50, in_place=in_place, weights_in_place=in_place)


def test_again_and_again():
    """A cache that grows by 20 rows and is cut back, five times, in place: the rows that survive are those of the plain form."""
    c = Case([300], 16, 32, 2, 2, BF16, seed=7)
    for _ in range(5):
        c.check(100, 4, 30, in_place=True, weights_in_place=False)
        c.w = c.rng.random(c.w.shape).astype(np.float32)
        c.lengths[:] = 120


def test_eviction_in_a_graph_on_another_stream():
    c = Case([500, 300], 16, 64, 2, 3, BF16, seed=8)
    table, lengths, into = (torch.tensor(x, device="cuda") for x in (c.table, c.lengths, c.into))
    w = torch.tensor(c.w, device="cuda")
    w_out, kept = torch.zeros_like(w), torch.zeros(3, 2, 2, 200, dtype=torch.int32, device="cuda")
    after = torch.zeros_like(lengths)
    call = lambda: c.cache.evict(table, lengths, w, 200, sink=4, recent=32, into=into, weights_out=w_out, kept=kept, lengths_out=after)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for k in range(3):
        w.copy_(torch.rand_like(w))
        call()
        torch.cuda.synchronize()
        want = [x.clone() for x in (kept, after, w_out, c.kp, c.vp)]
        kept.zero_(), after.zero_(), w_out.zero_()
        c.kp[:, c.into[:, :12].ravel()] = 0   # of the pages that rows go to, those they fill
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((kept, after, w_out, c.kp, c.vp), want))
