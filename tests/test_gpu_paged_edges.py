"""Calls of the paged cache where something unusual of one query, value or argument must stay with it, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paged_testlib import attention_error, f64, near
from paper_2605_22269_amd import binding as mk
from test_gpu_paged_attend import BF16, F32, Case, weights_error

pytestmark = pytest.mark.gpu


# ---- weights of rows beside a query whose scores are out of the ordinary ----
def window(D, dtype, causal_rows=300):
    """Two users' prompts whose bf16 form goes to the prompt kernel, and what a row's weight may be off."""
    c = Case([(32, causal_rows), (40, 200)], D, 28, 4, 16, dtype, seed=D)
    received = c.wanted()[1]
    return c, weights_error(c, received)


def weights_of(c):
    rows = torch.zeros(2, 4, int(c.lengths.max()), device="cuda")
    c.attend(weights_out=rows)
    return f64(rows)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_a_query_of_large_scores_leaves_its_neighbours_weights_alone(D, dtype):
    c, tol = window(D, dtype)
    c.q[2, 0] *= 2.0**30      # scores of 2^30 and more: one row has all of its weight
    received, got = c.wanted()[1], weights_of(c)
    for b, n in enumerate(c.lengths):
        near(got[b][:, :n], received[b], (1 + received[b]) * tol, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_an_infinite_score_stays_with_the_rows_that_its_query_sees(D, dtype):
    c, tol = window(D, dtype)
    past, token, row = 300 - 32, 3, 100
    at = (1, c.table[0][row // 16], slice(None), row % 16, 3)
    c.q[..., 3] = -1.0
    c.kp[at] = 30000.0        # a weight of nothing for everybody
    received = c.wanted()[1]
    c.kp[at] = float("inf")   # the same: -inf, but for one query
    c.q[token, 0, 3] = 1.0
    got = weights_of(c)
    unseen = slice(past + token + 1, 300)
    assert np.isnan(got[0][0, : past + token + 1]).all()
    near(got[0][:, unseen], received[0][:, unseen], (1 + received[0][:, unseen]) * tol, F32)
    near(got[0][1:, :300], received[0][1:], (1 + received[0][1:]) * tol, F32)
    near(got[1][:, :200], received[1], (1 + received[1]) * tol, F32)


# ---- threads ----
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_threads_on_streams_of_their_own_share_a_cache(dtype):
    """Each has its own sequences of the cache's pages, tables of its own width, and weights; the answers are those of one at a time."""
    import threading

    c = Case([(1, 300), (2, 77), (3, 1000), (40, 90), (1, 5), (6, 6)], 64, 8, 2, 16, dtype, seed=21)
    jobs = []
    for i in range(6):
        n, width = int(c.lengths[i]), -(-int(c.lengths[i]) // 16) + i
        table = np.full((1, width), -1, np.int32)
        table[0, : -(-n // 16)] = c.table[i, : -(-n // 16)]
        q = c.q[int(c.off[i]):int(c.off[i + 1])].contiguous()
        k, v = (torch.tensor(c.rng.standard_normal((q.shape[0], 2, 64)), dtype=torch.float32).to(dtype).cuda() for _ in "kv")
        jobs.append([torch.tensor(table, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"), q, k, v])

    def once(j):
        table, lengths, q, k, v = j
        w = torch.zeros(1, 2, int(c.lengths.max()), device="cuda")
        c.cache.append(1, table, lengths, k, v)
        return c.cache.attend(1, table, lengths, q, weights_out=w), w

    want = [once(j) for j in jobs]
    torch.cuda.synchronize()
    wrong, streams = [], [torch.cuda.Stream() for _ in jobs]

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(30):
                out, w = once(jobs[i])
                streams[i].synchronize()
                if not (torch.equal(out, want[i][0]) and torch.equal(w, want[i][1])):
                    wrong.append(i)

    all_of_them = [threading.Thread(target=work, args=(i,)) for i in range(6)]
    [t.start() for t in all_of_them]
    [t.join() for t in all_of_them]
    assert not wrong


def test_packed_sequences_of_no_tokens():
    q, k = (torch.empty(0, h, 64, dtype=BF16, device="cuda") for h in (4, 2))
    off, w = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((2, 2, 7), 5.0, device="cuda")
    for kw in ({}, dict(weights_out=w), dict(weights=w, weights_out=w, decay=0.5)):
        assert mk.PackedKV(n_q_heads=4).attend(q, k, k, off, **kw).shape == (0, 4, 64)
    assert (w == 5.0).all()   # rows past a sequence's length are left as they are


# ---- offsets that do not ascend ----
def test_offsets_that_overlap_leave_nothing_behind():
    """Tokens that are two sequences': more units than workgroups, of a tile some chunks and not others (tests/test_paged_offsets.py walks through
    it).  The next call on the same scratch is what it is on fresh scratch."""
    c = Case([(32, 128), (0, 50), (0, 384)], 64, 8, 1, 16, BF16, seed=30)
    table, lengths = torch.tensor(c.table, device="cuda"), torch.tensor(c.lengths, device="cuda")
    off = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    good, bad = off(0, 0, 0, 32), off(0, 32, 0, 32)
    fresh = mk.PagedKV(c.kp, c.vp, n_q_heads=8)
    want = fresh.attend(1, table, lengths, c.q, offsets=good)
    for _ in range(3):
        out = torch.full_like(c.q, 7.0)
        c.cache.attend(1, table, lengths, c.q, offsets=bad, out=out)
        assert (out == 7.0).all()
        assert torch.equal(c.cache.attend(1, table, lengths, c.q, offsets=good), want)
    c.news, c.off, c.lengths = np.array([0, 0, 32], np.int32), np.array([0, 0, 0, 32], np.int32), c.lengths
    c.check(want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_the_tokens_are_brought_inside(dtype):
    c = Case([(3, 40), (40, 300), (5, 64)], 64, 8, 1, 16, dtype, seed=31)
    want = c.attend()
    c.off[0], c.off[3] = -9, 2**31 - 1
    assert torch.equal(c.attend(), want)


# ---- values near the end of the range ----
@pytest.mark.parametrize("seqs,room", [([(150, 400), (60, 300)], 0), ([(150, 400), (60, 300)], 9000), ([(120, 5000)], 0), ([(3, 400), (1, 300)], 0)],
                         ids=["128", "256", "chunks", "few"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("high", [3.0, 8.0])
def test_the_largest_values_where_rows_decide_late(D, high, seqs, room):
    """Later rows' weights are far above 1 relative to the first rows' largest score, and the values so large that their products are past
    fp32, though no output is."""
    c = Case(seqs, D, 8, 2, 16, BF16, seed=D, width=-(-room // 16) if room else None)
    for b in range(len(seqs)):
        for j in range(40, int(c.lengths[b])):
            c.kp[:, c.table[b][j // 16], :, j % 16] *= high
    c.vp *= 1e35
    got, most = c.attend(), max(int(c.lengths.max()), 1)
    assert np.isfinite(f64(got)).all()
    want, _, amean, reach = c.wanted()
    near(f64(got), want, attention_error(amean, reach, most, D, BF16, True), BF16)
    rows = torch.zeros(len(seqs), 2, most, device="cuda")
    got, received = c.attend(weights_out=rows), c.wanted()[1]
    near(f64(got), want, attention_error(amean, reach, most, D, BF16, True), BF16)
    for b, n in enumerate(c.lengths):
        near(f64(rows)[b][:, :n], received[b], (1 + received[b]) * weights_error(c, received), F32)


# ---- outputs beside the weights of rows ----
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv", [(128, 28, 4), (64, 8, 1)])
@pytest.mark.parametrize("seqs,room", [([(16, 900), (40, 200), (0, 7)], 0), ([(300, 300), (200, 1000)], 9000), ([(120, 6000)], 0), ([(700, 5000)], 0),
                                       ([(1, 40), (2, 700)], 0)], ids=["window", "256", "chunks", "shares", "few"])
def test_asking_for_the_weights_changes_no_output(D, hq, hkv, seqs, room, dtype):
    c = Case(seqs, D, hq, hkv, 16, dtype, seed=40 + D, width=-(-room // 16) if room else None)
    rows = torch.zeros(len(seqs), hkv, int(c.lengths.max()), device="cuda")
    assert torch.equal(c.attend(weights_out=rows), c.attend())
    assert torch.isfinite(rows).all()
    for b, (new, n) in enumerate(seqs):   # what a query gives adds up to 1
        total, tokens = f64(rows)[b].sum(-1), new * hq // hkv
        assert (np.abs(total - tokens) <= (n + 64) * 2.0**-20 * max(tokens, 1)).all(), (total, tokens)
