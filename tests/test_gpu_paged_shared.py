"""Attention of groups of sequences that share rows, in 8 bits and not, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from batch_testlib import BF16, F32, Batch, i32
from paged_testlib import f64, near
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu
KINDS = [(BF16, False), (F32, False), (BF16, True), (F32, True)]
IDS = ["bf16", "f32", "bf16_8", "f32_8"]
SHAPES = [(128, 28, 4, 16), (64, 14, 2, 7), (32, 8, 8, 24), (16, 6, 1, 1)]
SETS = {  # sequences, groups
    "one": ([(1, 1)], [(1, 1)]),
    "users": ([(1, 30), (1, 1), (1, 500), (1, 77)], [(2, 900), (2, 33)]),
    "edges": ([(1, 31), (0, 5), (1, 0), (2, 2), (3, 129)], [(1, 0), (0, 64), (6, 128)]),       # no shared rows; a group of nobody; no own rows
    "long": ([(1, 5)] * 6, [(6, 9000)]),
    "few_and_many": ([(16, 16), (5, 90), (1, 700), (2, 2)], [(21, 40), (1, 2500), (2, 1)]),
}


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("D,hq,hkv,R", SHAPES)
@pytest.mark.parametrize("kind", SETS)
def test_shared_rows(D, hq, hkv, R, dtype, eight, kind):
    c = Batch(*SETS[kind], D, hq, hkv, R, dtype, eight, seed=D + R)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False), causal=False)


PROMPTS = {
    "questions": ([(n, n) for n in (9, 120, 33, 64)], [(226, 700)]),
    "past": ([(100, 300), (90, 1000), (1, 40)], [(190, 900), (1, 65)]),
    "few_own": ([(1, 1)] * 80, [(50, 2000), (30, 31)]),              # prompts to the shared rows, single tokens to their own
    "few_shared": ([(200, 200), (64, 70)], [(264, 1)]),
}


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 16), (64, 14, 2, 7), (128, 4, 4, 64)])
@pytest.mark.parametrize("room", [0, 9000])
@pytest.mark.parametrize("kind", PROMPTS)
def test_prompts(D, hq, hkv, R, eight, room, kind):
    c = Batch(*PROMPTS[kind], D, hq, hkv, R, BF16, eight, seed=D + R, shared_width=-(-room // R) if room else None)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)
    c.check(c.attend(causal=False, hint=300), causal=False)


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("D,hq,hkv,R", [(128, 28, 4, 32), (64, 4, 1, 5), (16, 32, 2, 16)])
@pytest.mark.parametrize("kind", ["users", "edges", "questions"])
def test_weights_of_own_and_shared_rows(D, hq, hkv, R, dtype, eight, kind):
    c = Batch(*{**SETS, **PROMPTS}[kind], D, hq, hkv, R, dtype, eight, seed=R + D)
    N, M = int(c.lengths.max()) + 5, int(c.shared_lengths.max()) + 3
    random = lambda *shape: torch.tensor(c.rng.random(shape), dtype=torch.float32, device="cuda")  # noqa: E731
    own, common = random(len(c.news), hkv, N), random(len(c.shared_lengths), hkv, M)
    own_out, common_out = torch.full_like(own, -3.0), torch.full_like(common, -3.0)
    out = c.attend(weights=own, weights_out=own_out, shared_weights=common, shared_weights_out=common_out, decay=0.5)
    assert torch.equal(out, c.attend())
    received, shared, reach = c.check(out)
    tol = c.weights_error(reach, c.T)
    for was, got, want, lengths in ((own, own_out, received, c.lengths), (common, common_out, shared, c.shared_lengths)):
        for b, n in enumerate(lengths):
            near(f64(got)[b][:, :n], 0.5 * f64(was)[b][:, :n] + want[b], (1 + want[b]) * tol, F32)
            assert (got[b, :, n:] == -3.0).all()
    one = torch.zeros_like(common)                                  # of the shared rows alone
    c.attend(shared_weights_out=one)
    other = torch.zeros_like(own)
    c.attend(weights_out=other)
    for got, want, lengths in ((one, shared, c.shared_lengths), (other, received, c.lengths)):
        for b, n in enumerate(lengths):
            near(f64(got)[b][:, :n], want[b], (1 + want[b]) * tol, F32)


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
def test_tokens_of_no_group_and_pages_that_are_none(dtype, eight):
    c = Batch([(2, 40), (1, 64), (3, 50), (70, 100)], [(3, 96), (2, 200)], 64, 4, 2, 8, dtype, eight, seed=8)
    c.shared_off[:] = [1, 3, 40]                                    # token 0 is nobody's, nor are those from 40 on
    c.shared_table[0, 3], c.shared_table[1, :4] = -1, c.n_pages
    c.table[2, :] = 2**31 - 1                                       # no row of their own
    c.shared_lengths[0] = 99999                                     # past the table
    for hint in (0, 70):
        c.check(c.attend(hint, max_new=hint))
    c.shared_lengths[:] = [-5, 2**31 - 1]
    c.check(c.attend())
    c.shared_off[:] = 0
    c.check(c.attend())
    c.shared_off[:] = [76, 76, 76]
    c.check(c.attend())


@pytest.mark.parametrize("users,hq,hkv,rows", [(16, 64, 1, 110000), (20, 56, 1, 64 * 1600), (3, 5, 1, 70000)])
def test_few_tiles_of_long_rows(users, hq, hkv, rows):
    """As many chunks of a tile as there can be."""
    c = Batch([(1, 3)] * users, [(users, rows)], 128, hq, hkv, 64, BF16, True, seed=3, layers=1, layer=0)
    first = c.attend()
    c.check(first)
    assert torch.equal(c.attend(), first)


@pytest.mark.parametrize("n", [70, 200])
def test_many_groups(n):
    rng = np.random.default_rng(n)
    sizes = rng.integers(0, 4, n)
    c = Batch([(int(m), int(m) + int(rng.integers(0, 30))) for m in sizes], [(int(m), int(rng.integers(0, 200))) for m in sizes], 32, 4, 2, 8, BF16, False, seed=n)
    c.check(c.attend())


@pytest.mark.parametrize("seqs", [[(1, 20), (1, 40), (1, 5)], [(70, 90), (64, 64), (1, 3)]])
def test_groups_whose_tokens_do_not_ascend_leave_outputs_as_they_are(seqs):
    c = Batch(seqs, [(0, 30), (0, 30), (0, 30)], 64, 8, 2, 16, BF16, False, seed=2)
    good = c.shared_off.copy()
    good[1:] = c.T
    c.shared_off[:] = [0, 2, 1, c.T]
    out = torch.full_like(c.q, 7.0)
    c.attend(out=out)
    assert (out == 7.0).all()
    c.shared_off[:] = good
    c.check(c.attend(out=out))                                      # and the workspace is fit for the next call
    c.off[1], c.off[2] = c.off[2], c.off[1]
    out.fill_(7.0)
    c.attend(out=out)
    assert (out == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("where", ["shared", "own"])
def test_scores_and_values_that_are_no_numbers(where, new, dtype):
    c = Batch([(new, new + 40), (new, new + 10)], [(new, 50), (new, 70)], 64, 4, 2, 16, dtype, False, seed=4)
    clean = c.attend()
    table = c.shared_table if where == "shared" else c.table
    at = (1, int(table[0][0]), slice(None), 3)
    for t, bad, nan in ((c.kp, float("nan"), True), (c.vp, float("inf"), False), (c.vp, float("nan"), True)):
        was = t[at].clone()
        t[at] = bad
        got = c.attend()
        assert torch.equal(got[new:], clean[new:])
        # (an infinity is multiplied by the two halves of a weight, the second of which may be negative or zero: infinite or a NaN)
        assert torch.isnan(got[:new]).all() if nan else not torch.isfinite(got[:new]).any()
        t[at] = was
    t = c.kp
    t[at] = -float("inf")                                           # -inf or +inf by the queries' sign: with positive ones a weight of zero
    c.q[:] = c.q.abs()
    assert torch.isfinite(c.attend()).all()


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("low,high", [(0.01, 100.0), (100.0, 0.01), (1e3, 1e3)])
@pytest.mark.parametrize("new", [1, 80])
def test_one_part_outweighs_the_other(low, high, new, dtype, eight):
    """Scores of shared rows of another size than those of own ones."""
    c = Batch([(new, 100 + new), (new, new)], [(2 * new, 150)], 64, 8, 2, 16, dtype, eight, seed=21)
    for table, by in ((c.shared_table, low), (c.table, high)):
        for page in table[table >= 0]:
            if eight:
                s = c.ks.view(torch.uint8)
                s[1, int(page)] = (s[1, int(page)].int() + int(np.round(np.log2(by)))).to(torch.uint8)
            else:
                c.kp[1, int(page)] *= by
    got = c.attend()
    want, _, _, amean, reach = c.wanted()
    sure = (c.D + 4) * 2.0**-24 * reach[..., 0] / 8 < 2.0**-4
    assert sure.any() and torch.isfinite(got).all()
    near(f64(got)[sure], want[sure], c.error(amean, reach)[sure], dtype)


def test_no_new_tokens():
    c = Batch([(0, 30), (0, 5)], [(0, 20)], 64, 4, 2, 8, BF16, False, seed=1)
    assert c.attend().shape == (0, 4, 64)
    w, s = torch.ones(2, 2, 30, device="cuda"), torch.ones(1, 2, 20, device="cuda")
    out, sout = torch.zeros_like(w), torch.zeros_like(s)
    c.attend(weights=w, weights_out=out, shared_weights=s, shared_weights_out=sout, decay=0.25)
    assert (out[0] == 0.25).all() and (out[1, :, :5] == 0.25).all() and (out[1, :, 5:] == 0).all() and (sout == 0.25).all()


@pytest.mark.parametrize("eight", [False, True])
def test_captured_and_replayed_beside_eager_calls(eight):
    c = Batch([(1, 300), (1, 2000), (1, 17)], [(2, 900), (1, 64)], 128, 8, 2, 16, BF16, eight, seed=30)
    table, lengths, group = i32(c.table), i32(c.lengths), c.group()
    out, eager = torch.empty_like(c.q), torch.empty_like(c.q)
    call = lambda o: c.cache.attend(1, table, lengths, c.q, out=o, shared=group)  # noqa: E731
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
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = call(torch.empty_like(c.q))
    torch.cuda.synchronize()
    assert torch.equal(other, out)


def test_equal_shares_need_no_offsets():
    c = Batch([(1, 30), (1, 60), (1, 9), (1, 2)], [(2, 100), (2, 50)], 128, 8, 2, 16, BF16, False, seed=31)
    plain = c.cache.attend(1, i32(c.table), i32(c.lengths), c.q, shared=mk.Shared(i32(c.shared_table), i32(c.shared_lengths)))
    c.check(plain)
    assert torch.equal(plain, c.attend())


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("D,new", [(64, 2), (128, 70), (64, 300)])
def test_padding_behind_the_sequences(D, new, dtype, eight):
    """Tokens of a group that are no sequence's are left as they are and count for no row's weight, whatever stands there."""
    c = Batch([(new, new + 70), (1, 40), (new, new + 5)], [(new, 90), (1 + new, 200)], D, 8, 2, 16, dtype, eight, seed=new + D)
    c.off[3] = c.off[2]                                             # the last sequence has none of its tokens
    n = int(c.off[2])
    for bad in (1e30, float("nan")):
        c.q[n:] = bad
        out = torch.full_like(c.q, 7.0)
        own = torch.zeros(3, 2, c.table.shape[1] * 16, device="cuda")
        common = torch.zeros(2, 2, c.shared_table.shape[1] * 16, device="cuda")
        c.attend(out=out, weights_out=own, shared_weights_out=common)
        assert (out[n:] == 7.0).all()
        c.q[n:] = 0
        want, received, shared, amean, reach = c.wanted()
        near(f64(out)[:n], want[:n], c.error(amean, reach)[:n], dtype)
        tol = c.weights_error(reach, c.T)
        for got, want, lengths in ((own, received, c.lengths), (common, shared, c.shared_lengths)):
            for b, m in enumerate(lengths):
                near(f64(got)[b][:, :m], want[b], (1 + want[b]) * tol, F32)
