"""Shared rows of caches whose rows lie apart give what those of dense ones give."""
import pytest
import torch

from batch_testlib import BF16, F32, Batch
from paged_testlib import on_device
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,slack", [(BF16, 8), (F32, 4)])
@pytest.mark.parametrize("order", ["page_head_row", "page_row_head"])
@pytest.mark.parametrize("seqs,groups", [([(1, 30), (1, 1), (1, 500)], [(2, 900), (1, 33)]), ([(120, 300), (100, 140)], [(220, 700)])])
def test_rows_that_lie_apart(seqs, groups, order, dtype, slack):
    c = Batch(seqs, groups, 64, 14, 2, 16, dtype, False, seed=6)
    dense = c.attend()
    c.check(dense)
    apart = [on_device(t.float().cpu().numpy(), dtype, order, slack) for t in (c.kp, c.vp)]
    assert all(t.stride()[3 if order == "page_head_row" else 2] == 64 + slack for t in apart)
    c.cache = mk.PagedKV(*apart, n_q_heads=14)
    assert torch.equal(c.attend(), dense)
