"""The paged cache's calls together, as examples/conversation.py uses them."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from paged_testlib import attention, attention_error, f64, gathered, near  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_conversation(dtype):
    import conversation

    steps, budget, layers, hkv = 5, 60, 2, 2
    talk, out, asked, kept = conversation.run(users=3, layers=layers, q_heads=6, kv_heads=hkv, head_dim=64, retrieved=40,
                                              questions=(3, 50, 17), steps=steps, window=8, budget=budget, dtype=dtype, seed=3)
    want = [min(n + 40, budget) + steps for n in (3, 50, 17)]
    assert talk.rows == want and talk.lengths.tolist() == want
    used = talk.table[talk.table >= 0].tolist()
    assert len(set(used)) == len(used) and sorted(used + talk.free) == list(range(talk.k_pages.shape[1]))
    for b, n in enumerate((3, 50, 17)):     # nothing of a short conversation goes, the first and last rows never do
        rows = kept[:, b].cpu().numpy()
        m = min(n + 40, budget)
        assert (np.diff(rows[..., :m]) > 0).all() and (rows[..., m:] == -1).all()
        assert (rows[..., :4] == np.arange(4)).all() and (rows[..., m - 1] == n + 39).all()
    k, v, table = f64(talk.k_pages), f64(talk.v_pages), talk.table.cpu().numpy()
    for layer in range(layers):             # the last step's outputs are the attention over the rows that are there now
        def rows_of(b, n):
            kk, ok = gathered(k, layer, table, want, 16, b, n)
            return kk, gathered(v, layer, table, want, 16, b, n)[0], ok

        ref, _, amean, reach = attention(f64(asked[layer]), rows_of, want, [0, 1, 2, 3], hkv, True, table.shape[1] * 16)
        near(f64(out[layer]), ref, attention_error(amean, reach, max(want), 64, dtype), dtype)
        w = talk.weights[layer].cpu().numpy()
        for b in range(3):
            assert (w[b, :, : want[b]] >= 0).all() and (w[b, :, want[b]:] == 0).all() and (w[b, :, want[b] - 1] > 0).all()
