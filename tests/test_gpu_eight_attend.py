"""Attention over a paged cache in 8 bits against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from batch_testlib import BF16, F32, Batch, i32
from paged_testlib import f64, near
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu
SHAPES = [  # D, query heads, KV heads, page rows
    (128, 28, 4, 16), (64, 14, 2, 7), (32, 8, 8, 24), (16, 6, 1, 1), (128, 5, 5, 64), (64, 64, 2, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", SHAPES)
@pytest.mark.parametrize("seqs", [
    [(1, 1)], [(1, 500)], [(1, 31), (1, 32), (1, 33), (1, 0), (1, 129)], [(16, 16), (5, 900), (0, 40), (1, 2)],
    [(3, 2), (2, 0), (4, 3001)]], ids=["one", "some", "edges", "mixed", "short_and_long"])
def test_attention_over_pages(D, hq, hkv, R, dtype, seqs):
    c = Batch(seqs, None, D, hq, hkv, R, dtype, True, seed=D + R + len(seqs))
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 16), (64, 14, 2, 7), (128, 4, 4, 64), (64, 8, 1, 1), (128, 12, 1, 24)])
@pytest.mark.parametrize("seqs", [[(300, 300)], [(37, 1000), (256, 257), (0, 10), (60, 31), (129, 129)], [(100, 6001)], [(70, 64), (64, 2000), (500, 500)]],
                         ids=["whole", "mixed", "past", "edges"])
@pytest.mark.parametrize("room", [0, 9000])
def test_prompts(D, hq, hkv, R, seqs, room):
    c = Batch(seqs, None, D, hq, hkv, R, BF16, True, seed=D + R + len(seqs), width=-(-room // R) if room else None)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("seqs", [[(300, 900)], [(1600, 6400)], [(64, 64), (200, 500)]])
def test_prompts_are_bit_for_bit_those_over_what_the_rows_stand_for(seqs):
    c = Batch(seqs, None, 128, 8, 2, 16, BF16, True, seed=5)
    k, v = (torch.tensor(x).to(BF16).cuda() for x in c.values())
    plain = mk.PagedKV(k, v, n_q_heads=8).attend(c.layer, i32(c.table), i32(c.lengths), c.q, offsets=i32(c.off))
    assert torch.equal(c.attend(), plain)


@pytest.mark.parametrize("order", ["page_row_head", "head_page_row"])
def test_orders_of_the_pages_and_strided_queries(order):
    c = Batch([(3, 77), (1, 300)], None, 64, 8, 2, 16, BF16, True, seed=5, order=order)
    wide = torch.full((4, 20, 64), 9.0, dtype=BF16, device="cuda")
    wide[:, 6:14] = c.q
    c.q = wide[:, 6:14]
    c.check(c.attend())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,news,rows,room", [(64, 6, 50, 0), (128, 16, 40, 0), (16, 3, 3, 0), (32, 5, 90, 0), (64, 200, 230, 0), (128, 130, 140, 0),
                                              (64, 400, 401, 5000), (128, 230, 260, 5000)])
def test_hidden_rows_and_scales_never_reach_a_token(D, news, rows, room, dtype):
    """What only the last token sees is no number; past the last row nothing was ever written, scales are any bytes, and so is the first
    page of the layer, where rows that live nowhere are read."""
    c = Batch([(news, rows), (news, rows)], None, D, 4, 2, 16, dtype, True, seed=D + news, width=-(-room // 16) if room else None)
    c.lengths[1] = rows - 1
    c.table[1, 0] = -1
    clean = c.attend()
    page, r = c.table[0][(rows - 1) // 16], (rows - 1) % 16
    for t, s in ((c.kp.view(torch.uint8), c.ks.view(torch.uint8)), (c.vp.view(torch.uint8), c.vs.view(torch.uint8))):
        t[1, page, :, r, ::3] = 0x7F
        t[1, page, :, r + 1:] = 0xFF
        s[1, page, :, r + 1:] = 255
        s[1, c.table[1][(rows - 1) // 16], :, r:] = 255
        free = [p for p in range(c.n_pages) if p not in c.table]
        t[1, free], s[1, free] = 0x7E, 255
    got = c.attend()
    last = c.off[1] - 1
    assert torch.equal(got[:last], clean[:last]) and torch.equal(got[c.off[1]:], clean[c.off[1]:])
    assert not torch.isfinite(got[last]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_that_are_none_and_rows_past_the_table(dtype):
    c = Batch([(2, 96), (1, 64), (3, 50), (1, 10), (80, 90)], None, 64, 4, 2, 8, dtype, True, seed=8, width=12)
    c.lengths[0] = 110
    c.table[1, 3] = -1
    c.table[1, 0] = c.n_pages
    c.table[2, :] = 2**31 - 1
    c.table[3, 1] = -(2**31)
    c.table[4, 5] = -3
    for hint in (0, 80):
        c.check(c.attend(max_new=hint))
    assert not f64(c.attend())[c.off[2]:c.off[3]].any()
    c.check(c.attend(causal=False), causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_rows_are_shared_out_and_joined(dtype):
    c = Batch([(1, 20011)], None, 128, 8, 1, 16, dtype, True, seed=1)
    first = c.attend()
    c.check(first)
    for _ in range(3):
        assert torch.equal(c.attend(), first)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 32), (64, 4, 1, 5), (32, 6, 6, 16), (16, 32, 2, 16)])
@pytest.mark.parametrize("seqs", [[(1, 700)], [(16, 333), (3, 2), (0, 12), (1, 0), (2, 1500)], [(60, 300), (90, 90)]], ids=["one", "mixed", "prompts"])
def test_weights_that_rows_receive(D, hq, hkv, R, seqs, dtype):
    c = Batch(seqs, None, D, hq, hkv, R, dtype, True, seed=R + D)
    c.table[0, 2] = -1
    N = int(c.lengths.max()) + 5
    before = torch.tensor(c.rng.random((len(seqs), hkv, N)), dtype=torch.float32, device="cuda")
    after = torch.full_like(before, -3.0)
    out = c.attend(weights=before, weights_out=after, decay=0.5)
    assert torch.equal(out, c.attend())
    received, _, reach = c.check(out)
    tol = c.weights_error(reach, int(c.news.max()))
    for b, n in enumerate(c.lengths):
        was, got = f64(before)[b], f64(after)[b]
        near(got[:, :n], 0.5 * was[:, :n] + received[b], (1 + received[b]) * tol, F32)
        assert (got[:, n:] == -3.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_very_different_sizes(dtype):
    """Scales from the smallest to large ones, keys of 2^20 and of 2^-60 side by side."""
    c = Batch([(4, 200), (70, 300)], None, 64, 8, 2, 16, dtype, True, seed=3)
    for s, lo, hi in ((c.ks, 60, 122), (c.vs, 10, 150)):
        s.view(torch.uint8)[:] = torch.tensor(c.rng.integers(lo, hi, s.shape), dtype=torch.uint8, device="cuda")
    for hint in (1, 70):
        c.check(c.attend(max_new=hint))


def test_captured_and_replayed_beside_eager_calls():
    c = Batch([(1, 300), (1, 2000), (1, 17)], None, 128, 8, 2, 16, BF16, True, seed=30)
    table, lengths = i32(c.table), i32(c.lengths)
    out, eager = torch.empty_like(c.q), torch.empty_like(c.q)
    call = lambda o: c.cache.attend(1, table, lengths, c.q, out=o)  # noqa: E731
    call(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(5):
        c.q.normal_()
        lengths -= 1
        graph.replay()
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


@pytest.mark.parametrize("new", [2, 300])
def test_offsets_far_past_32_bits(new):
    """Pages, and their scales, that lie past 4 GiB: written, attended to alone and as what others share."""
    D, R, n = 128, 1024, 34000
    kp, vp = (torch.zeros(1, n, 1, R, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv")
    big = torch.zeros(n, 130 * 1024, dtype=torch.uint8, device="cuda")
    scales = [big.as_strided((1, n, 1, R), (0, 130 * 1024, 0, 1), storage_offset=x) for x in (0, 2048)]
    far = mk.PagedKV8(kp, vp, *scales, n_q_heads=8)
    near_by = Batch([(new, 1500)], None, D, 8, 1, R, BF16, True, seed=4, layers=1, layer=0)
    table, lengths, off = i32([[n - 1, n - 2]]), i32([1500]), i32([0, new])
    k, v = (torch.randn(1500, 1, D, device="cuda").bfloat16() for _ in "kv")
    far.append(0, table, lengths, k, v)
    near_by.cache.append(0, i32(near_by.table), lengths, k, v)
    assert torch.equal(far.attend(0, table, lengths, near_by.q, offsets=off), near_by.attend())
    own = torch.randn(new, 1, D, device="cuda").bfloat16()
    far.append(0, i32([[n - 5]]), i32([new]), own, own)
    spare = i32([[p for p in range(near_by.n_pages) if p not in near_by.table][:1]])
    near_by.cache.append(0, spare, i32([new]), own, own)
    a = far.attend(0, i32([[n - 5]]), i32([new]), near_by.q, offsets=off, shared=mk.Shared(table, lengths))
    b = near_by.cache.attend(0, spare, i32([new]), near_by.q, offsets=off, shared=mk.Shared(i32(near_by.table), lengths))
    assert torch.equal(a, b)


def test_no_new_tokens():
    c = Batch([(0, 30), (0, 5)], None, 64, 4, 2, 8, BF16, True, seed=1)
    assert c.attend().shape == (0, 4, 64)
    w = torch.ones(2, 2, 30, device="cuda")
    out = torch.zeros_like(w)
    c.attend(weights=w, weights_out=out, decay=0.25)
    assert (out[0] == 0.25).all() and (out[1, :, :5] == 0.25).all() and (out[1, :, 5:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("power", [-100, -60, 60, 100])
def test_queries_and_rows_of_far_sizes(power, dtype):
    """Queries times 2^power, keys times 2^-power: scores, and with them outputs, stay what they are.  (Of an fp32 query of 2^-100 the last part
    may be less than the least normal number: 2^-126 2^100 of a key's size, 2^-2 of a rounding of a score, may be lost.)"""
    c = Batch([(1, 500), (5, 60)], None, 128, 8, 2, 16, dtype, True, seed=9)
    first = c.attend()
    c.q *= 2.0**power
    c.ks.view(torch.uint8)[:] -= power if power > 0 else power + 256
    got = c.attend()
    c.check(got)
    assert torch.equal(got, first) or (dtype == F32 and power == -100)
