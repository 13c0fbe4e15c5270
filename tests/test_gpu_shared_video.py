"""The cache in 8 bits and shared rows together, as examples/shared_video.py uses them."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from batch_testlib import Batch  # noqa: E402
from paged_testlib import f64, near  # noqa: E402

pytestmark = pytest.mark.gpu


class Seen(Batch):
    """The last step of the example, as a batch of the tests."""

    def __init__(self, rooms, layer, q):
        cpu = lambda t: t.cpu().numpy()  # noqa: E731
        self.table, self.lengths, self.shared_table, self.shared_lengths = (cpu(t) for t in (rooms.table, rooms.lengths, rooms.video_table, rooms.video_lengths))
        self.kp, self.vp, self.ks, self.vs = rooms.k_pages, rooms.v_pages, rooms.k_scales, rooms.v_scales
        self.news, self.off = np.ones(len(self.lengths), np.int32), np.arange(len(self.lengths) + 1, dtype=np.int32)
        self.shared_off = np.concatenate([[0], np.cumsum(rooms.users)]).astype(np.int32)
        self.T, self.hq, self.D = q.shape
        _, self.n_pages, self.hkv, self.R, _ = rooms.k_pages.shape
        self.layer, self.q, self.dtype, self.eight, self.grouped = layer, q, q.dtype, True, True


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_rooms(dtype, head_dim):
    import shared_video

    steps, budget, layers = 3, 40, 2
    rooms, out, asked, kept = shared_video.run(users_of_room=(3, 1, 2), video_rows=(300, 17, 90), layers=layers, q_heads=6, kv_heads=2, head_dim=head_dim,
                                               question=(3, 70), steps=steps, budget=budget, dtype=dtype, seed=3)
    asked_tokens = [3 + 7 * b for b in range(6)]
    want = [min(n, budget) + steps for n in asked_tokens]
    assert rooms.rows == want and rooms.lengths.tolist() == want
    for b, n in enumerate(asked_tokens):
        rows, m = kept[:, b].cpu().numpy(), min(n, budget)
        assert (np.diff(rows[..., :m]) > 0).all() and (rows[..., m:] == -1).all() and (rows[..., min(m, 4) - 1] == min(m, 4) - 1).all()
    for layer in range(layers):
        c = Seen(rooms, layer, asked[layer])
        ref, _, _, amean, reach = c.wanted()
        near(f64(out[layer]), ref, c.error(amean, reach), dtype)
        w = rooms.weights[layer].cpu().numpy()
        for b in range(6):
            assert (w[b, :, : want[b]] > 0).all() and (w[b, :, want[b]:] == 0).all()
