"""What attention over shared rows leaves for the call's other launch, where a group holds few of many single tokens and its rows are long: no tile
in more chunks than the other launch has room for."""
import pytest
import torch

from batch_testlib import BF16, Batch
from paged_testlib import f64, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("D,hq,hkv,users,group,rows", [(64, 14, 2, 1280, 18, 140000), (128, 8, 1, 2200, 48, 110000)])
def test_a_group_of_few_among_many(D, hq, hkv, users, group, rows, eight):
    c = Batch([(1, 1 + i % 40) for i in range(users)], [(group, rows)], D, hq, hkv, 64, BF16, eight, seed=5, layers=1, layer=0)
    first = c.attend(hint=group, max_new=1)
    c.check(first)
    assert torch.equal(c.attend(hint=group, max_new=1), first)
    common = torch.zeros(1, hkv, rows, device="cuda")
    assert torch.equal(c.attend(hint=group, max_new=1, shared_weights_out=common), first)
    _, _, shared, _, reach = c.wanted()
    near(f64(common)[0], shared[0], (1 + shared[0]) * c.weights_error(reach, group), torch.float32)
