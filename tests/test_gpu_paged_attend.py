"""Attention over a paged cache and over packed sequences, and the weights rows receive, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paged_testlib import attention, attention_error, f64, gathered, near, on_device, spread_tables
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Case:
    """Sequences of (new tokens, rows) in a paged cache of random values."""

    def __init__(self, seqs, D, hq, hkv, R, dtype, seed, order="page_head_row", layers=2, layer=1, q_scale=1.5, width=None):
        rng = self.rng = np.random.default_rng(seed)
        self.news, self.lengths = (np.array(x, np.int32) for x in zip(*seqs))
        self.D, self.hq, self.hkv, self.R, self.dtype, self.layer = D, hq, hkv, R, dtype, layer
        self.table, self.n_pages = spread_tables(rng, self.lengths, R, width)
        shape = (layers, self.n_pages, hkv, R, D)
        self.kp, self.vp = (on_device(rng.standard_normal(shape).astype(np.float32), dtype, order) for _ in "kv")
        self.off = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)
        self.q = torch.tensor(rng.standard_normal((int(self.off[-1]), hq, D)) * q_scale, dtype=torch.float32).to(dtype).cuda()
        self.cache = mk.PagedKV(self.kp, self.vp, n_q_heads=hq)

    def attend(self, **kw):
        t = [torch.tensor(x, device="cuda") for x in (self.table, self.lengths, self.off)]
        return self.cache.attend(self.layer, t[0], t[1], self.q, offsets=t[2], **kw)

    def wanted(self, causal=True):
        k, v = f64(self.kp), f64(self.vp)

        def rows(b, n):
            kk, ok = gathered(k, self.layer, self.table, self.lengths, self.R, b, n)
            return kk, gathered(v, self.layer, self.table, self.lengths, self.R, b, n)[0], ok

        return attention(f64(self.q), rows, self.lengths, self.off, self.hkv, causal, self.table.shape[1] * self.R)

    def check(self, got, causal=True):
        # more than a token or two a sequence: rows of 64 and 128 bf16 features are multiplied by weights of 8 bits
        single_weights = self.dtype == BF16 and self.D >= 64 and -(-int(self.off[-1]) // len(self.news)) * (self.hq // self.hkv) >= 48
        want, received, amean, reach = self.wanted(causal)
        near(f64(got), want, attention_error(amean, reach, max(self.lengths.max(), 1), self.D, self.dtype, single_weights), self.dtype)
        return received


def weights_error(c, received):
    """Of a row's weight, which adds up at most n_new * G of them, each off as in attention_error (of values of 1)."""
    _, _, _, reach = c.wanted()
    worst = reach.max() if reach.size else 0.0
    rel = attention_error(1.0, worst, max(c.lengths.max(), 1), c.D, F32) + (2 * (c.D + 4) * 2.0**-24 * worst / np.sqrt(c.D) if c.dtype == BF16 else 0)
    return rel + 2.0**-23 * max(1, c.news.max() * (c.hq // c.hkv)) / 16


SHAPES = [  # D, query heads, KV heads, page rows
    (128, 28, 4, 16), (64, 14, 2, 7), (32, 8, 8, 24), (16, 6, 1, 1), (128, 5, 5, 64), (64, 64, 2, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", SHAPES)
@pytest.mark.parametrize("seqs", [
    [(1, 1)], [(1, 500)], [(1, 31), (1, 32), (1, 33), (1, 0), (1, 129)], [(16, 16), (5, 900), (0, 40), (1, 2)],
    [(3, 2), (2, 0), (4, 3000)]], ids=["one", "some", "edges", "mixed", "short_and_long"])
def test_attention_over_pages(D, hq, hkv, R, dtype, seqs):
    c = Case(seqs, D, hq, hkv, R, dtype, seed=D + R + len(seqs))
    c.check(c.attend())
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 16), (64, 14, 2, 7), (128, 4, 4, 64), (64, 8, 1, 1), (128, 12, 1, 24)])
@pytest.mark.parametrize("seqs", [[(300, 300)], [(37, 1000), (256, 257), (0, 10), (60, 31), (129, 129)], [(100, 6001)], [(70, 64), (64, 2000), (500, 500)]],
                         ids=["whole", "mixed", "past", "edges"])
@pytest.mark.parametrize("room", [0, 9000])   # how many rows the table has room for decides between tiles of 128 and 256 queries
def test_prompts(D, hq, hkv, R, seqs, room):
    c = Case(seqs, D, hq, hkv, R, BF16, seed=D + R + len(seqs), width=-(-room // R) if room else None)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False), causal=False)


def test_prompts_over_pages_that_are_none():
    c = Case([(200, 300), (90, 90), (150, 64)], 128, 8, 2, 16, BF16, seed=14)
    c.table[0, 3], c.table[0, 17] = -1, 2**31 - 1
    c.table[2, :] = -5
    c.check(c.attend())
    c.check(c.attend(causal=False), causal=False)


def test_prompts_with_scores_of_any_size():
    c = Case([(100, 100), (70, 900)], 64, 4, 2, 16, BF16, seed=16, q_scale=1e17)
    got, want = f64(c.attend()), c.wanted()[0]
    # (one row each, but for scores nearer than 64 terms' rounding of themselves)
    assert (np.abs(got - want).max(-1) <= 2.0**-6 * np.abs(want).max()).mean() > 0.999
    c = Case([(100, 100)], 64, 4, 2, 16, BF16, seed=17)
    c.q[3, 1, 7], c.q[50, 2] = float("nan"), -float("inf")
    got = f64(c.attend())
    bad = ~np.isfinite(got).all(-1)
    assert np.isnan(got[3, 1]).all() and np.isnan(got[50, 2]).all() and bad.sum() == 2


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("low,high,at", [(0.02, 60.0, 150), (60.0, 0.02, 150), (1.0, 400.0, 299), (1e-3, 1e4, 40)])
def test_scores_that_grow_or_fall_by_much_along_the_rows(low, high, at, D, dtype):
    """Rows from `at` on have keys of another size: what exponents subtract at first is far from the largest score of all."""
    c = Case([(200, 300), (40, 200)], D, 8, 2, 16, dtype, seed=D + at, width=300 if at == 150 else None)
    for b in range(2):
        for j in range(int(c.lengths[b])):
            c.kp[:, c.table[b][j // 16], :, j % 16] *= low if j < at else high
    want, _, amean, reach = c.wanted()
    got = c.attend()
    # a score this large is known to its own rounding only: where that is less than a sixteenth
    err = attention_error(amean, reach, 300, D, dtype, dtype == BF16)
    sure = (D + 4) * 2.0**-24 * reach[..., 0] / np.sqrt(D) < 2.0**-4
    assert sure.any() or high > 1e3   # (there only that the outputs are numbers)
    near(f64(got)[sure], want[sure], err[sure], dtype)
    assert np.isfinite(f64(got)).all()


@pytest.mark.parametrize("causal", [True, False])
def test_prompts_whose_first_page_is_none(causal):
    c = Case([(150, 400), (150, 150)], 128, 8, 2, 64, BF16, seed=18, width=100)
    c.table[:, 0] = -1
    c.kp[:] *= 40.0     # scores of a few hundred, either sign: the rows that are there decide what exponents subtract
    want, _, amean, reach = c.wanted(causal)
    err = attention_error(amean, reach, 400, 128, BF16, True)
    near(f64(c.attend(causal=causal)), want, err, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_rows_are_shared_out_and_joined(dtype):
    c = Case([(1, 20011)], 128, 8, 1, 16, dtype, seed=1)
    first = c.attend()
    c.check(first)
    for _ in range(3):   # the order of the sums does not depend on who finishes first
        assert torch.equal(c.attend(), first)
    c = Case([(2, 9000), (1, 17), (1, 0), (7, 4000)], 64, 12, 4, 48, dtype, seed=2)
    c.check(c.attend())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [64, 65, 200])
def test_many_sequences(dtype, n):
    rng = np.random.default_rng(n)
    c = Case([(int(rng.integers(0, 3)), int(rng.integers(0, 300))) for _ in range(n)], 32, 4, 2, 8, dtype, seed=n)
    c.check(c.attend())


@pytest.mark.parametrize("order", ["page_row_head", "head_page_row"])
def test_orders_of_the_pages_and_strided_queries(order):
    c = Case([(3, 77), (1, 300)], 64, 8, 2, 16, BF16, seed=5, order=order)
    wide = torch.full((4, 20, 64), 9.0, dtype=BF16, device="cuda")
    wide[:, 6:14] = c.q
    c.q = wide[:, 6:14]
    c.check(c.attend())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,hq,hkv", [(128, 14, 2), (64, 4, 1), (16, 3, 3)])
def test_packed_sequences(D, hq, hkv, causal, dtype):
    rng = np.random.default_rng(D)
    news = [1, 0, 37, 128, 5, 260]
    off = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    T = int(off[-1])
    qkv = torch.tensor(rng.standard_normal((T, hq + 2 * hkv, D)), dtype=torch.float32).to(dtype).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    got = mk.PackedKV(n_q_heads=hq).attend(q, k, v, torch.tensor(off, device="cuda"), causal=causal)
    kk, vv = f64(k), f64(v)
    rows = lambda b, n: (kk[off[b]:off[b + 1]], vv[off[b]:off[b + 1]], np.ones(n, bool))
    want, _, amean, reach = attention(f64(q), rows, news, off, hkv, causal, T)
    near(f64(got), want, attention_error(amean, reach, 260, D, dtype, single_weights=True), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_that_are_none_and_rows_past_the_table(dtype):
    c = Case([(2, 96), (1, 64), (3, 50), (1, 10)], 64, 4, 2, 8, dtype, seed=8, width=12)
    c.lengths[0] = 110              # its table ends at 96: what follows does not exist, but counts
    c.table[1, 3] = -1
    c.table[1, 0] = c.n_pages
    c.table[2, :] = 2**31 - 1       # no row at all: zeros
    c.table[3, 1] = -(2**31)
    c.check(c.attend())
    assert not f64(c.attend())[c.off[2]:c.off[3]].any()
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_lengths_that_make_no_sense_are_brought_in_range(dtype):
    c = Case([(2, 40), (1, 40), (5, 20)], 32, 2, 1, 8, dtype, seed=9)
    c.lengths[:] = [2**31 - 1, -7, 3]
    c.check(c.attend())
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,news,rows,room", [(64, 6, 50, 0), (128, 16, 40, 0), (16, 3, 3, 0), (64, 200, 230, 0), (128, 130, 140, 0), (128, 33, 33, 0),
                                              (64, 400, 401, 5000), (128, 230, 260, 5000)])
def test_hidden_rows_never_reach_a_token(D, news, rows, room, dtype, bad):
    """The last row's key and value are no numbers: only the last token sees it.  So is what lies past the last row, and on the first
    page of the layer, where rows that live nowhere are read."""
    c = Case([(news, rows), (news, rows)], D, 4, 2, 16, dtype, seed=D + news, width=-(-room // 16) if room else None)
    c.lengths[1] = rows - 1
    c.table[1, 0] = -1
    clean = c.attend()
    page, r = c.table[0][(rows - 1) // 16], (rows - 1) % 16
    for t in (c.kp, c.vp):
        t[1, page, :, r, ::3] = bad
        t[1, page, :, r + 1:] = bad
        t[1, c.table[1][(rows - 1) // 16], :, r:] = bad
    free = [p for p in range(c.n_pages) if p not in c.table]
    c.kp[1, free], c.vp[1, free] = bad, bad
    got = c.attend()
    last = c.off[1] - 1
    assert torch.equal(got[:last], clean[:last]) and torch.equal(got[c.off[1]:], clean[c.off[1]:])
    assert not torch.isfinite(got[last]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_first_page_of_the_layer_holds_no_numbers(dtype):
    """Rows that live nowhere are read from page 0."""
    c = Case([(1, 20), (4, 9)], 64, 4, 2, 16, dtype, seed=3)
    swap = np.where(c.table == 0, c.n_pages - 1, np.where(c.table == c.n_pages - 1, 0, c.table))
    keep = (c.table == 0).any()
    k0, v0 = c.kp.clone(), c.vp.clone()
    if keep:
        for t, o in ((c.kp, k0), (c.vp, v0)):
            t[:, c.n_pages - 1] = o[:, 0]
        c.table = np.where(c.table == 0, c.n_pages - 1, c.table).astype(np.int32)
    c.table[1, 0] = -1
    want = c.attend()
    c.kp[:, 0], c.vp[:, 0] = float("nan"), float("inf")
    assert torch.equal(c.attend(), want) and torch.isfinite(want).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinite_and_absent_scores(dtype):
    c = Case([(1, 40), (1, 40), (1, 40)], 64, 2, 1, 8, dtype, seed=4)
    c.q[0, 0, 5] = float("nan")
    row = lambda b, j: (1, c.table[b][j // 8], 0, j % 8)
    c.kp[row(1, 17)] = float("inf")
    c.q[1] = c.q[1].abs()                     # +inf
    c.kp[row(2, 3)] = -float("inf")
    c.q[2] = c.q[2].abs()                     # -inf: a weight of zero
    got = f64(c.attend())
    assert np.isnan(got[0, 0]).all() and np.isfinite(got[0, 1]).all() and np.isnan(got[1]).all() and np.isfinite(got[2]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_any_finite_size(dtype):
    """Scores far past where exponentials overflow: the largest takes all."""
    c = Case([(1, 100), (2, 5000)], 64, 4, 2, 16, dtype, seed=6, q_scale=1e17)
    got = f64(c.attend())
    want = c.wanted()[0]
    assert np.abs(got - want).max() <= 2.0**-6 * np.abs(want).max()   # (one row each, but for scores nearer than 2^-24 of themselves)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 32), (64, 4, 1, 5), (32, 6, 6, 16), (16, 32, 2, 16)])
@pytest.mark.parametrize("seqs", [[(1, 700)], [(16, 333), (3, 2), (0, 12), (1, 0), (2, 1500)]], ids=["one", "mixed"])
def test_weights_that_rows_receive(D, hq, hkv, R, seqs, dtype):
    c = Case(seqs, D, hq, hkv, R, dtype, seed=R + D)
    c.table[0, 2] = -1
    N = int(c.lengths.max()) + 5
    before = torch.tensor(c.rng.random((len(seqs), hkv, N)), dtype=torch.float32, device="cuda")
    first, after = before.clone(), torch.full_like(before, -3.0)
    out = c.attend(weights=before, weights_out=after, decay=0.5)
    assert torch.equal(out, c.attend())
    received = c.check(out)
    tol = weights_error(c, received)
    for b, n in enumerate(c.lengths):
        was, got = f64(before)[b], f64(after)[b]
        near(got[:, :n], 0.5 * was[:, :n] + received[b], (1 + received[b]) * tol, F32)
        assert (got[:, n:] == -3.0).all()
    assert torch.equal(before, first)
    fresh = torch.full_like(before, 8.0)
    c.attend(weights_out=fresh)                                       # from nothing
    for b, n in enumerate(c.lengths):
        near(f64(fresh)[b][:, :n], received[b], (1 + received[b]) * tol, F32)
    c.attend(weights=fresh, weights_out=fresh)                        # in place, accumulating
    for b, n in enumerate(c.lengths):
        near(f64(fresh)[b][:, :n], 2 * received[b], (2 + 2 * received[b]) * tol, F32)
    # fewer rows than the sequences have: the others' weights are nobody's
    short = torch.full((len(seqs), hkv, 100), 5.0, device="cuda")
    c.attend(weights_out=short[:, :, :40])
    for b, n in enumerate(c.lengths):
        near(f64(short)[b][:, : min(n, 40)], received[b][:, :40], (1 + received[b][:, :40]) * tol, F32)
    assert (short[:, :, 40:] == 5.0).all()


@pytest.mark.parametrize("D,hq,hkv,R,new", [(128, 28, 4, 16, 16), (64, 64, 8, 7, 16), (128, 8, 1, 64, 60)])
def test_weights_of_windows_of_many_users(D, hq, hkv, R, new):
    c = Case([(new, 300), (new, new), (new, new - 5), (new, 1700), (new, 90), (new, 64)], D, hq, hkv, R, BF16, seed=R + D)
    c.table[0, 2] = -1
    N = int(c.lengths.max()) + 5
    got = torch.full((6, hkv, N), -3.0, device="cuda")
    received = c.check(c.attend(weights_out=got, max_new=new))
    again = torch.zeros_like(got)
    c.attend(weights_out=again, max_new=new)
    tol = weights_error(c, received)
    for b, n in enumerate(c.lengths):
        near(f64(got)[b][:, :n], received[b], (1 + received[b]) * tol, F32)
        assert (got[b, :, n:] == -3.0).all() and torch.equal(again[b, :, :n], got[b, :, :n])


def test_hints_choose_kernels_and_nothing_else():
    """The longest sequence is longer than the hint says, or far shorter."""
    c = Case([(1, 500), (40, 700), (0, 3), (300, 310)], 128, 28, 4, 16, BF16, seed=20)
    for hint in (0, 1, 5, 1000):
        c.check(c.attend(max_new=hint))


def test_no_new_tokens():
    c = Case([(0, 30), (0, 5)], 64, 4, 2, 8, BF16, seed=1)
    assert c.attend().shape == (0, 4, 64)
    w = torch.ones(2, 2, 30, device="cuda")
    out = torch.zeros_like(w)
    c.attend(weights=w, weights_out=out, decay=0.25)
    assert (out[0] == 0.25).all() and (out[1, :, :5] == 0.25).all() and (out[1, :, 5:] == 0).all()


def test_offsets_past_32_bits():
    """A layer whose pages lie more than 4 GB apart."""
    R, D = 16, 128
    big = torch.zeros(3 * (1 << 30), dtype=BF16, device="cuda")   # 6 GB
    step = 1 << 30                                               # 2 GB between pages
    strides = (0, step, R * D, D, 1)
    rng = np.random.default_rng(2)
    kp, vp = big.as_strided((1, 3, 1, R, D), strides), big[1 << 20:].as_strided((1, 3, 1, R, D), strides[:1] + strides[1:])
    for t in (kp, vp):
        t.copy_(torch.tensor(rng.standard_normal(t.shape), dtype=torch.float32).to(BF16))
    c = Case.__new__(Case)
    c.rng, c.news, c.lengths, c.off = rng, np.array([1], np.int32), np.array([45], np.int32), np.array([0, 1], np.int32)
    c.D, c.hq, c.hkv, c.R, c.dtype, c.layer, c.n_pages, c.kp, c.vp = D, 4, 1, R, BF16, 0, 3, kp, vp
    c.table = np.array([[2, 0, 1]], np.int32)
    c.q = torch.tensor(rng.standard_normal((1, 4, D)), dtype=torch.float32).to(BF16).cuda()
    c.cache = mk.PagedKV(kp, vp, n_q_heads=4)
    c.check(c.attend())


def test_on_another_stream_and_in_a_graph():
    c = Case([(1, 400), (2, 4000)], 128, 8, 2, 16, BF16, seed=12)
    want = c.attend()
    args = [torch.tensor(x, device="cuda") for x in (c.table, c.lengths, c.off)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = c.cache.attend(1, args[0], args[1], c.q, offsets=args[2])
    side.synchronize()
    assert torch.equal(got, want)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.stream(side):   # the workspace of the capturing stream is there before
        c.cache.attend(1, args[0], args[1], c.q, offsets=args[2], out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c.cache.attend(1, args[0], args[1], c.q, offsets=args[2], out=out)
    for k in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        c.q.mul_(1.0 + 0.5 * (k % 2))
        want = c.attend()
        torch.cuda.synchronize()


def test_graphs_whose_replays_come_in_any_order():
    """Two graphs captured on one stream, nothing run on it before: the second's first replay comes before any of the first's, and
    eager calls on that stream, larger than both, in between."""
    c = Case([(1, 400), (2, 4000)], 128, 8, 2, 16, BF16, seed=12)
    want = c.attend()
    args = [torch.tensor(x, device="cuda") for x in (c.table, c.lengths, c.off)]
    torch.cuda.synchronize()
    side, graphs, outs = torch.cuda.Stream(), [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        outs.append(torch.zeros_like(want))
        with torch.cuda.graph(graphs[-1], stream=side):
            for _ in range(2):
                c.cache.attend(1, args[0], args[1], c.q, offsets=args[2], out=outs[-1])
    for k in (1, 0, 1, 1, 0):
        outs[k].zero_()
        torch.cuda.synchronize()
        graphs[k].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[k], want)
        got = torch.zeros_like(want)
        w = torch.zeros(2, 2, 4000, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c.cache.attend(1, args[0], args[1], c.q, offsets=args[2], out=got, weights_out=w)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def wanted_of_one(c, causal=True):
    """Case.wanted of a single long sequence, in float64 on the device, a head at a time."""
    n, new = int(c.lengths[0]), int(c.off[1])
    at = torch.arange(n, device="cuda")
    page = torch.tensor(c.table, device="cuda")[0].long()[at // c.R]
    there = (page >= 0) & (page < c.kp.shape[1])
    k, v = (x[c.layer][page.clamp(0, x.shape[1] - 1), :, at % c.R].double() for x in (c.kp, c.vp))
    seen = there[None].expand(new, n)
    if causal:
        seen = seen & (at[None] <= n - new + torch.arange(new, device="cuda")[:, None])
    outs, received = [], torch.zeros(c.hkv, n, dtype=torch.float64, device="cuda")
    for h in range(c.hq):
        g = h * c.hkv // c.hq
        kk, vv, q = k[:, g].contiguous(), torch.where(there[:, None], v[:, g], 0.0).contiguous(), c.q[:, h].double()
        w = torch.softmax((q @ kk.T / np.sqrt(c.D)).masked_fill(~seen, -np.inf), -1)
        received[g] += w.sum(0)
        reach = (q.abs() @ kk.abs().T).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        outs.append([x.cpu().numpy() for x in (w @ vv, w @ vv.abs(), reach)])
    out, amean, reach = (np.stack(x, 1) for x in zip(*outs))
    return out, [received.cpu().numpy()], amean, reach


def one_long(D, hq, hkv, new, past, seed):
    c = Case([(new, new + past)], D, hq, hkv, 24, BF16, seed=seed)
    c.wanted = lambda causal=True: wanted_of_one(c, causal)
    return c


@pytest.mark.parametrize("D,hq,hkv,new,past", [(128, 64, 8, 590, 4410), (128, 28, 4, 1568, 4000), (64, 28, 4, 1568, 6272), (128, 12, 12, 1500, 3001)])
def test_one_long_prompt(D, hq, hkv, new, past):
    """One sequence with somewhat fewer tiles than compute units, or somewhat more: its rows are shared out evenly, tile after tile."""
    c = one_long(D, hq, hkv, new, past, new)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False), causal=False)
    c.table[0, 5], c.table[0, 121] = -1, 2**31 - 1
    rows = torch.zeros(1, hkv, new + past, device="cuda")
    received = c.check(c.attend(weights_out=rows))
    near(f64(rows)[0], received[0], (1 + received[0]) * weights_error(c, received), F32)


def test_one_long_prompt_with_rows_that_decide_late():
    c = one_long(128, 28, 4, 1568, 4000, 19)
    n = 5568
    for j in range(n):
        c.kp[:, c.table[0][j // 24], :, j % 24] *= 0.02 if j < 4300 else 30.0
    bad = slice(None), c.table[0][(n - 5) // 24], slice(None), (n - 5) % 24
    c.vp[bad] = float("inf")   # seen by the last five tokens
    c.q[:300] = 0.0
    got = f64(c.attend())
    assert np.isfinite(got[:-5]).all()
    c.vp[bad] = 0.0
    want, _, amean, reach = c.wanted()
    err = attention_error(amean, reach, n, 128, BF16, True)
    sure = (128 + 4) * 2.0**-24 * reach[..., 0] / np.sqrt(128) < 2.0**-4
    sure[-5:] = False
    assert sure.any()
    near(got[sure], want[sure], err[sure], BF16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("high", [3.0, 8.0])
def test_large_values_where_rows_decide_late(D, high):
    """Weights are relative to the first rows' largest score at first: later ones far above it must not take large values out of range."""
    c = Case([(150, 400), (60, 300)], D, 8, 2, 16, BF16, seed=D)
    for b in range(2):
        for j in range(40, int(c.lengths[b])):
            c.kp[:, c.table[b][j // 16], :, j % 16] *= high
    c.vp *= 1e30
    got = c.attend()
    assert np.isfinite(f64(got)).all()
    want, _, amean, reach = c.wanted()
    near(f64(got), want, attention_error(amean, reach, 400, D, BF16, True), BF16)
