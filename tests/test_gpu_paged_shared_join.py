"""Own rows and shared ones whose scores lie so far apart that one part's factor is zero where they are joined: what the lesser part holds that is no
number still reaches the tokens that see it, as it does where all rows are the sequence's own."""
import pytest
import torch

from batch_testlib import BF16, F32, Batch
from paged_testlib import f64, near

pytestmark = pytest.mark.gpu
KINDS = [(BF16, False), (F32, False), (BF16, True), (F32, True)]
IDS = ["bf16", "f32", "bf16_8", "f32_8"]
LESS = 3   # row of the lesser part that is looked at


def apart(new, dtype, eight, lesser, D, rows=150):
    """Two sequences of a group each.  Scores of the lesser part are about zero, those of the other 128 and more (in log2 units past 180: a weight
    of the lesser part, 2^-180 of the whole, is zero in fp32)."""
    c = Batch([(new, new + 40)] * 2, [(new, rows)] * 2, D, 8, 2, 16, dtype, eight, seed=new + D)
    c.q[:] = c.q.abs().clamp(min=1.0)
    large = c.table if lesser == "shared" else c.shared_table
    for table in (c.table, c.shared_table):
        for page in table[table >= 0]:
            if eight:   # the sign away, and the power of two made one that is
                c.kp.view(torch.uint8)[1, int(page)] = 0x38     # 1
                c.ks.view(torch.uint8)[1, int(page)] = 127 + 5 if table is large else 0x7F - 30
            else:
                c.kp[1, int(page)] = 32.0 if table is large else 2.0**-30
    return c


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("new,D", [(1, 64), (1, 128), (80, 64), (80, 128), (300, 128), (3, 16)])
@pytest.mark.parametrize("lesser", ["shared", "own"])
def test_what_is_no_number_counts_however_little_it_weighs(lesser, new, D, dtype, eight):
    c = apart(new, dtype, eight, lesser, D)
    clean = c.attend()
    assert torch.isfinite(clean).all()
    c.check(clean)
    table = c.shared_table if lesser == "shared" else c.table
    at = (1, int(table[0][0]), slice(None), LESS)
    nan = 0x7F if eight else float("nan")
    for t, bad in ((c.kp, nan), (c.vp, nan), *([] if eight else [(c.vp, float("inf"))])):
        rows = t.view(torch.uint8) if eight else t
        was = rows[at].clone()
        rows[at] = bad
        got = c.attend()
        assert torch.equal(got[new:], clean[new:])              # the other sequence's
        if eight or bad != bad:
            assert torch.isnan(got[:new]).all()
        else:
            assert not torch.isfinite(got[:new]).any()
        # with the rows' weights: a score that is no number makes them none
        common = torch.zeros(2, 2, 150, device="cuda")
        own = torch.zeros(2, 2, new + 40, device="cuda")
        again = c.attend(weights_out=own, shared_weights_out=common)
        assert torch.equal(torch.isnan(again), torch.isnan(got)) and torch.equal(again[new:], got[new:])
        if t is c.kp:
            assert torch.isnan(common[0]).all() and torch.isnan(own[0, :, :40]).all()
        assert torch.isfinite(common[1]).all() and torch.isfinite(own[1]).all()
        rows[at] = was
    assert torch.equal(c.attend(), clean)


@pytest.mark.parametrize("dtype,eight", KINDS, ids=IDS)
@pytest.mark.parametrize("new", [1, 80])
@pytest.mark.parametrize("lesser", ["shared", "own"])
def test_rows_that_are_not_there_count_for_nothing(lesser, new, dtype, eight):
    """A part of no rows at all, beside one of large scores: what stands in pages that nobody names reaches nobody."""
    c = apart(new, dtype, eight, lesser, 64)
    (c.shared_table if lesser == "shared" else c.table)[0] = -1
    clean = c.attend()
    assert torch.isfinite(clean).all()
    want, _, _, amean, reach = c.wanted()
    near(f64(clean), want, c.error(amean, reach), dtype)
    table = c.shared_table if lesser == "shared" else c.table
    named = {int(p) for t in (c.table, c.shared_table) for p in t[t >= 0]}
    spare = [p for p in range(c.n_pages) if p not in named]
    assert spare and table is not None
    for t in (c.kp, c.vp):
        rows = t.view(torch.uint8) if eight else t
        rows[1, spare] = 0x7F if eight else float("nan")
    assert torch.equal(c.attend(), clean)
