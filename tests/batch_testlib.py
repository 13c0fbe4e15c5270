"""Batches of sequences over a paged cache, in 8 bits or not, with rows that groups of them share or without, and what attention over them
gives in 64 bits."""
import numpy as np
import torch

from eight_testlib import random_cache, stands_for
from paged_testlib import attention_error, f64, near, on_device, places, spread_tables
from paper_2605_22269_amd import binding as mk

BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Batch:
    """seqs: (new tokens, rows) of each; groups: (new tokens, rows that are shared) of each, or None."""

    def __init__(self, seqs, groups, D, hq, hkv, R, dtype, eight, seed, order="page_head_row", layers=2, layer=1, q_scale=1.5, width=None,
                 shared_width=None):
        rng = self.rng = np.random.default_rng(seed)
        self.news, self.lengths = (np.array(x, np.int32) for x in zip(*seqs))
        self.D, self.hq, self.hkv, self.R, self.dtype, self.layer, self.eight = D, hq, hkv, R, dtype, layer, eight
        self.off = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)
        self.T = int(self.off[-1])
        common = [n for _, n in groups] if groups else []
        both, self.n_pages = spread_tables(rng, [*self.lengths, *common], R, max([-(-int(n) // R) for n in (*self.lengths, *common)] + [1, width or 0, shared_width or 0]))
        n = len(seqs)
        need = lambda x, w: max([-(-int(m) // R) for m in x] + [1, w or 0])  # noqa: E731
        self.table = np.ascontiguousarray(both[:n, : need(self.lengths, width)])
        self.grouped = groups is not None
        if self.grouped:
            self.shared_table = np.ascontiguousarray(both[n:, : need(common, shared_width)])
            self.shared_lengths = np.array(common, np.int32)
            self.shared_off = np.concatenate([[0], np.cumsum([m for m, _ in groups])]).astype(np.int32)
        shape = (layers, self.n_pages, hkv, R, D)
        if eight:
            self.kp, self.vp, self.ks, self.vs = random_cache(rng, shape, spread=0, order=order)
            self.cache = mk.PagedKV8(self.kp, self.vp, self.ks, self.vs, n_q_heads=hq, dtype=dtype)
        else:
            self.kp, self.vp = (on_device(rng.standard_normal(shape).astype(np.float32), dtype, order) for _ in "kv")
            self.cache = mk.PagedKV(self.kp, self.vp, n_q_heads=hq)
        self.q = torch.tensor(rng.standard_normal((self.T, hq, D)) * q_scale, dtype=torch.float32).to(dtype).cuda()

    def values(self):
        if self.eight:
            return stands_for(self.kp, self.ks), stands_for(self.vp, self.vs)
        return f64(self.kp), f64(self.vp)

    def group(self, **kw):
        return mk.Shared(i32(self.shared_table), i32(self.shared_lengths), i32(self.shared_off), **kw)

    def attend(self, hint=0, **kw):
        if self.grouped and "shared" not in kw:
            kw["shared"] = self.group(max_tokens=hint)
        return self.cache.attend(self.layer, i32(self.table), i32(self.lengths), self.q, offsets=i32(self.off), **kw)

    def wanted(self, causal=True):
        """Outputs, what own and shared rows receive, the mean of |v| under an output's weights, the largest sum |q_i k_i|."""
        k, v = (x[self.layer] for x in self.values())
        G, D = self.hq // self.hkv, self.D
        q = f64(self.q)
        out, amean, reach = np.zeros_like(q), np.zeros_like(q), np.zeros((self.T, self.hq, 1))
        room = self.table.shape[1] * self.R
        rows = lambda table, lengths, b, n: places(table, lengths, self.R, self.n_pages, b, np.arange(n))  # noqa: E731
        common, shared_got = [], []
        if self.grouped:
            for g in range(len(self.shared_lengths)):
                n = min(max(int(self.shared_lengths[g]), 0), self.shared_table.shape[1] * self.R)
                common.append(rows(self.shared_table, self.shared_lengths, g, n))
                shared_got.append(np.zeros((self.hkv, n)))
        received = []
        for b in range(len(self.lengths)):
            lo, hi = int(self.off[b]), int(self.off[b + 1])
            length = max(int(self.lengths[b]), 0)
            n = min(length, room)
            page, r, ok = rows(self.table, self.lengths, b, n)
            own = np.zeros((self.hkv, n))
            for i in range(hi - lo):
                t = lo + i
                seen = ok & (np.arange(n) <= length - (hi - lo) + i) if causal else ok
                p, rr, g, some = page[seen], r[seen], -1, np.zeros(0, bool)
                if self.grouped:
                    owner = [x for x in range(len(common)) if self.shared_off[x] <= t < self.shared_off[x + 1]]
                    if owner:
                        g = owner[0]
                        cp, cr, some = common[g]
                        p, rr = np.concatenate([cp[some], p]), np.concatenate([cr[some], rr])
                if not len(p):
                    continue
                m = int(some.sum())
                for h in range(self.hkv):
                    qq, kk, vv = q[t, h * G:(h + 1) * G], k[p, h, rr], v[p, h, rr]
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = qq @ kk.T / np.sqrt(D)
                        w = np.exp(s - s.max(-1, keepdims=True))
                        w = w / w.sum(-1, keepdims=True)
                        out[t, h * G:(h + 1) * G], amean[t, h * G:(h + 1) * G] = w @ vv, w @ np.abs(vv)
                        reach[t, h * G:(h + 1) * G] = (np.abs(qq) @ np.abs(kk).T).max(-1, keepdims=True)
                    got = w.sum(0)
                    own[h, seen] += got[m:]
                    if g >= 0:
                        shared_got[g][h, some] += got[:m]
            received.append(own)
        return out, received, shared_got, amean, reach

    def rows_seen(self):
        n = max(min(int(self.lengths.max()), self.table.shape[1] * self.R), 1)   # (no more than a table has room for)
        return n + (min(max(int(self.shared_lengths.max()), 0), self.shared_table.shape[1] * self.R) if self.grouped else 0)

    def of_parts(self, reach):
        """fp32 over rows in 8 bits, relative, on top of attention_error: queries and weights are three bf16, of at most 1, 2^-7 and 2^-15 of
        them, and 32 products of each add up in the matrix core: 32 (1 + 2^-7 + 2^-15) + 3 < 36 roundings and two where four such sums are
        joined, for the 12 of a score there, in numerator and denominator; 36 and one where a block of 32 rows joins the rest, for the
        20 of sums over rows."""
        return (2 * (38 - 12) * reach / np.sqrt(self.D) + (37 - 20)) * 2.0**-24 if self.eight and self.dtype == F32 else 0.0

    def error(self, amean, reach):
        """paged_testlib.attention_error, and for the join of own rows with shared ones: the difference of two references (each at most as
        large as a score) and a multiplication and an addition more."""
        G = self.hq // self.hkv
        most = max(self.T // max(len(self.news), 1), int(self.news.max()), int(np.diff(self.shared_off).max()) if self.grouped else 0)
        single = self.dtype == BF16 and self.D >= 64 and most * G >= 48
        err = attention_error(amean, reach, self.rows_seen(), self.D, self.dtype, single) + amean * self.of_parts(reach)
        return err + amean * (8 + 4 * 1.4427 * reach / np.sqrt(self.D)) * 2.0**-24 if self.grouped else err

    def check(self, got, causal=True):
        want, own, common, amean, reach = self.wanted(causal)
        near(f64(got), want, self.error(amean, reach), self.dtype)
        return own, common, reach

    def weights_error(self, reach, tokens):
        """Of a row's weight, relative: each of those that add up is off as in error() (of values of 1), and they are added up."""
        worst = reach.max() if reach.size else 0.0
        rel = attention_error(1.0, worst, self.rows_seen(), self.D, F32) + (2 * (self.D + 4) * 2.0**-24 * worst / np.sqrt(self.D) if self.dtype == BF16 else 0)
        rel = rel + self.of_parts(worst)
        return rel + (8 + 4 * 1.4427 * worst / np.sqrt(self.D)) * 2.0**-24 + 2.0**-23 * max(1, tokens * (self.hq // self.hkv)) / 16
