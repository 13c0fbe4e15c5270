"""A conversation about a video, for several users at once, on the paged cache.

    python examples/conversation.py            # sizes of the 7B head layout, random weights

Every user first gets a prompt: the rows that a retrieval found in the video's cache (they are keys and values already and are
only placed), then the question's tokens.  When a user's cache grows past its budget it is cut back to the rows that the
last tokens looked at.  Then the users' answers are generated together, a token a step.  The model around the attention is left
out: what its projections would yield is drawn at random.
"""
from __future__ import annotations

import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_22269_amd import binding as mk  # noqa: E402


class Conversation:
    """Pages of all layers, a table and a length per user, the weight every row has received; which pages are free."""

    def __init__(self, users, *, layers, q_heads, kv_heads, head_dim, page_rows=16, max_rows=2048, budget=1024, sink=4, recent=64,
                 dtype=torch.bfloat16, device="cuda"):
        self.users, self.layers, self.page_rows, self.budget, self.sink = users, layers, page_rows, budget, sink
        self.recent = min(recent, (budget - sink) // 2)     # of a small budget half is left to the weights
        width = -(-max_rows // page_rows)
        shape = (layers, users * width, kv_heads, page_rows, head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=dtype, device=device) for _ in "kv")
        self.cache = mk.PagedKV(self.k_pages, self.v_pages, n_q_heads=q_heads)
        self.weights = torch.zeros(layers, users, kv_heads, max_rows, device=device)
        self.table = torch.full((users, width), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(users, dtype=torch.int32, device=device)
        self.rows = [0] * users                             # the lengths, on the host
        self.free = list(range(users * width))[::-1]
        pair = torch.arange(head_dim // 2, device=device)
        # time, height and width take the frequencies in turn
        self.rope = mk.Rope(1e4 ** (-2.0 * pair.double() / head_dim), (pair % 3).to(torch.int32), n_axes=3)

    def grow(self, new):
        """Room for new[b] more rows of every user; the lengths count them from here on."""
        for b, n in enumerate(new):
            have, need = -(-self.rows[b] // self.page_rows), -(-(self.rows[b] + n) // self.page_rows)
            if need > have:
                pages = [self.free.pop() for _ in range(need - have)]
                self.table[b, have:need] = torch.tensor(pages, dtype=torch.int32, device=self.table.device)
            self.rows[b] += n
        self.lengths.copy_(torch.tensor(self.rows, dtype=torch.int32))

    def place(self, layer, k, v, offsets):
        """Rows that are keys and values already ([tokens][KV head][feature], any strides), the last ones that grow() counted."""
        self.cache.append(layer, self.table, self.lengths, k, v, offsets=offsets)

    def tokens(self, layer, q, k, v, positions, offsets=None, max_new=1):
        """New tokens at one layer: rotated, placed, and attending to their users' rows."""
        q = self.cache.append(layer, self.table, self.lengths, k, v, q=q, offsets=offsets, rope=self.rope, positions=positions)
        w = self.weights[layer]
        if max_new > 16:   # a prompt: what rows are worth is what its last tokens look at (look_back)
            return self.cache.attend(layer, self.table, self.lengths, q, offsets=offsets, max_new=max_new), q
        return self.cache.attend(layer, self.table, self.lengths, q, offsets=offsets, max_new=max_new, weights=w, weights_out=w), q

    def look_back(self, layer, q_last, offsets, window):
        """The weights of all rows from the (rotated) queries of the users' last `window` tokens."""
        self.cache.attend(layer, self.table, self.lengths, q_last, offsets=offsets, max_new=window, weights_out=self.weights[layer])

    def cut_back(self):
        """Users past their budget are brought back to it, in place; their last pages are free again.  Returns the rows kept."""
        kept, _ = self.cache.evict(self.table, self.lengths, self.weights, self.budget, sink=self.sink, recent=self.recent,
                                   lengths_out=self.lengths)
        for b in range(self.users):
            have, need = -(-self.rows[b] // self.page_rows), -(-min(self.rows[b], self.budget) // self.page_rows)
            if need < have:
                self.free += self.table[b, need:have].tolist()
                self.table[b, need:have] = -1
            self.rows[b] = min(self.rows[b], self.budget)
        return kept


def offsets_of(new):
    o = [0]
    for n in new:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device="cuda")


def run(users=4, layers=28, q_heads=28, kv_heads=4, head_dim=128, retrieved=700, questions=(20, 333, 900, 61), steps=32, window=16,
        budget=1024, dtype=torch.bfloat16, seed=0):
    """Returns the conversation, the last step's outputs and queries per layer, and what was kept."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    talk = Conversation(users, layers=layers, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, budget=budget, dtype=dtype)
    new = list(questions[:users])
    past = [retrieved] * users
    talk.grow(past)
    where = offsets_of(past)
    for layer in range(layers):   # gathered rows stand [KV head][row][feature]: placed as they stand
        k, v = (normal(kv_heads, retrieved * users, head_dim).transpose(0, 1) for _ in "kv")
        talk.place(layer, k, v, where)
    talk.grow(new)
    where, T = offsets_of(new), sum(new)
    at = torch.cat([torch.arange(n, device="cuda") + m for n, m in zip(new, past)])
    positions = at.to(torch.int32).expand(3, T).contiguous()   # text: the same position on every axis
    last = [min(window, n) for n in new]
    for layer in range(layers):
        qkv = normal(T, q_heads + 2 * kv_heads, head_dim)
        _, q = talk.tokens(layer, qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], qkv[:, q_heads + kv_heads:], positions, where, max(new))
        ends = where.tolist()
        talk.look_back(layer, torch.cat([q[ends[b + 1] - last[b]:ends[b + 1]] for b in range(users)]), offsets_of(last), window)
    kept = talk.cut_back()
    out, asked = [None] * layers, [None] * layers
    for step in range(steps):
        talk.grow([1] * users)
        positions = torch.tensor([n + retrieved + step for n in new], dtype=torch.int32, device="cuda").expand(3, users).contiguous()
        for layer in range(layers):
            qkv = normal(users, q_heads + 2 * kv_heads, head_dim)
            out[layer], asked[layer] = talk.tokens(layer, qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], qkv[:, q_heads + kv_heads:],
                                                   positions)
    return talk, out, asked, kept


def main():
    run(steps=2)   # the first pass loads kernels and takes scratch
    torch.cuda.synchronize()
    begin = time.perf_counter()
    talk, _, _, _ = run(steps=64)
    torch.cuda.synchronize()
    print(f"4 users, 28 layers: prompts of 20 to 900 tokens over 700 retrieved rows, cut back, 64 steps: {time.perf_counter() - begin:.3f} s;"
          f" rows now {talk.rows}, {len(talk.free)} pages free")


if __name__ == "__main__":
    main()
