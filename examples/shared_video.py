"""Several users in several rooms, each room watching a video of its own: the video's rows lie in the cache once, in 8 bits.

    python examples/shared_video.py            # sizes of the 7B head layout, random weights

A room's video is prefilled first: its keys and values go to pages of the room (rotated on the way, in 8 bits).  Every user then has
rows of their own, questions and answers, behind what the room shares; all users' new tokens attend in one call a layer, the room's
rows once for all of its users.  Users' rows are cut back to a budget by the weight they received.  The model around the
attention is left out: what its projections would yield is drawn at random.
"""
from __future__ import annotations

import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_22269_amd import binding as mk  # noqa: E402


def i32(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def offsets_of(n):
    o = [0]
    for x in n:
        o.append(o[-1] + x)
    return i32(o)


class Rooms:
    """The cache of all rooms and users.  Users of a room are next to each other."""

    def __init__(self, users_of_room, video_rows, *, layers, q_heads, kv_heads, head_dim, page_rows=16, max_rows=1024, budget=512, dtype=torch.bfloat16):
        self.users, self.video_rows, self.page_rows, self.budget = users_of_room, video_rows, page_rows, budget
        n_users = sum(users_of_room)
        per_video, per_user = [-(-n // page_rows) for n in video_rows], -(-max_rows // page_rows)
        n_pages = sum(per_video) + n_users * per_user
        shape = (layers, n_pages, kv_heads, page_rows, head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv")
        self.k_scales, self.v_scales = (torch.zeros(shape[:4], dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in "kv")
        self.cache = mk.PagedKV8(self.k_pages, self.v_pages, self.k_scales, self.v_scales, n_q_heads=q_heads, dtype=dtype)
        at, rows = 0, []
        for n in per_video:
            rows.append(list(range(at, at + n)) + [-1] * (max(per_video) - n))
            at += n
        self.video_table, self.video_lengths = i32(rows), i32(video_rows)
        self.table = torch.arange(at, n_pages, dtype=torch.int32, device="cuda").view(n_users, per_user).contiguous()
        self.lengths, self.rows = i32([0] * n_users), [0] * n_users
        self.weights = torch.zeros(layers, n_users, kv_heads, max_rows, device="cuda")
        pair = torch.arange(head_dim // 2, device="cuda")
        self.rope = mk.Rope(1e4 ** (-2.0 * pair.double() / head_dim), (pair % 3).to(torch.int32), n_axes=3)

    def watch(self, layer, k, v, positions):
        """Keys and values of all rooms' videos, one after the other."""
        self.cache.append(layer, self.video_table, self.video_lengths, k, v, offsets=offsets_of(self.video_rows), rope=self.rope, positions=positions)

    def grow(self, new):
        """Room for new[b] more rows of every user; who shares what is worked out once for all layers."""
        self.rows = [a + b for a, b in zip(self.rows, new)]
        self.lengths.copy_(i32(self.rows))
        self.offsets, self.most = offsets_of(new), max(new)
        tokens, at = [], 0
        for n in self.users:
            tokens.append(sum(new[at:at + n]))
            at += n
        self.shared = mk.Shared(self.video_table, self.video_lengths, offsets_of(tokens), max_tokens=max(tokens))

    def tokens(self, layer, q, k, v, positions):
        """New tokens at one layer: rotated, written, and attending to their room's video and their user's rows."""
        q = self.cache.append(layer, self.table, self.lengths, k, v, q=q, offsets=self.offsets, rope=self.rope, positions=positions)
        w = self.weights[layer]
        return self.cache.attend(layer, self.table, self.lengths, q, offsets=self.offsets, max_new=self.most, weights=w, weights_out=w,
                                 shared=self.shared), q

    def cut_back(self):
        kept, _ = self.cache.evict(self.table, self.lengths, self.weights, self.budget, sink=4, recent=min(64, (self.budget - 4) // 2),
                                   lengths_out=self.lengths)
        self.rows = [min(n, self.budget) for n in self.rows]
        return kept


def run(users_of_room=(20, 12, 16), video_rows=(6272, 2000, 4100), layers=28, q_heads=28, kv_heads=4, head_dim=128, question=(5, 60), steps=16,
        budget=512, dtype=torch.bfloat16, seed=0):
    """Returns the rooms, the last step's outputs and queries per layer, and what was kept."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    rooms = Rooms(users_of_room, list(video_rows), layers=layers, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, budget=budget, dtype=dtype)
    at = torch.cat([torch.arange(n, device="cuda") for n in video_rows])
    grid = torch.stack([at // 196, at % 196 // 14, at % 14]).to(torch.int32).contiguous()   # frames of 14 x 14 tokens
    for layer in range(layers):
        kv = normal(sum(video_rows), 2 * kv_heads, head_dim)
        rooms.watch(layer, kv[:, :kv_heads], kv[:, kv_heads:], grid)
    n_users = sum(users_of_room)
    new = [question[0] + (7 * b) % (question[1] - question[0] + 1) for b in range(n_users)]
    out, asked, kept = [None] * layers, [None] * layers, None
    for step in range(steps + 1):
        rooms.grow(new)
        T = sum(new)
        positions = torch.cat([torch.arange(n - m, n) for n, m in zip(rooms.rows, new)]).add_(7000).to("cuda", torch.int32).expand(3, T).contiguous()
        for layer in range(layers):
            qkv = normal(T, q_heads + 2 * kv_heads, head_dim)
            out[layer], asked[layer] = rooms.tokens(layer, qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], qkv[:, q_heads + kv_heads:], positions)
        if step == 0:
            kept = rooms.cut_back()
        new = [1] * n_users
    return rooms, out, asked, kept


def main():
    run(steps=2)   # the first pass loads kernels and takes scratch
    torch.cuda.synchronize()
    begin = time.perf_counter()
    rooms, _, _, _ = run(steps=64)
    torch.cuda.synchronize()
    print(f"48 users in 3 rooms, 28 layers: videos of {rooms.video_rows} rows, questions of 5 to 60 tokens, 64 steps:"
          f" {time.perf_counter() - begin:.3f} s; a page of 16 rows in 8 bits is {rooms.k_pages[0, 0].numel() * 2 + rooms.k_scales[0, 0].numel() * 2} bytes")


if __name__ == "__main__":
    main()
