"""Rows written to a paged cache in 8 bits, and read back, against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from eight_testlib import codes, exponents, held, random_cache, stands_for
from paged_testlib import f64, near, places, rotated, rotation_error, spread_tables
from paper_2605_22269_amd import binding as mk

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Written:
    """A cache, and new tokens of every sequence for it."""

    def __init__(self, seed, news, lengths, D, hq, hkv, R, dtype, order="page_head_row", layers=2, slack=0):
        rng = self.rng = np.random.default_rng(seed)
        self.news, self.lengths, self.R, self.dtype, self.D, self.hkv, self.hq = news, lengths, R, dtype, D, hkv, hq
        self.table, n_pages = spread_tables(rng, np.maximum(lengths, 1), R)
        self.kp, self.vp, self.ks, self.vs = random_cache(rng, (layers, n_pages, hkv, R, D), order=order, slack=slack)
        self.cache = mk.PagedKV8(self.kp, self.vp, self.ks, self.vs, n_q_heads=hq, dtype=dtype)
        self.off = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.T = int(self.off[-1])
        qkv = torch.tensor(rng.standard_normal((self.T, hq + 2 * hkv, D)), dtype=torch.float32).to(dtype)
        qkv[:, hq:] *= torch.tensor(np.exp2(rng.integers(-30, 30, (self.T, 2 * hkv, 1)))).to(dtype)
        self.qkv = qkv.cuda()
        self.q, self.k, self.v = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]

    def before(self):
        return [t.clone() for t in (self.kp.view(torch.uint8), self.vp.view(torch.uint8), self.ks.view(torch.uint8), self.vs.view(torch.uint8))]

    def rows(self):
        """(sequence, token, page, row in it, is there) of every new token."""
        for b, n in enumerate(self.news):
            page, r, ok = places(self.table, self.lengths, self.R, self.kp.shape[1], b, np.arange(self.lengths[b] - n, self.lengths[b]))
            for i in range(n):
                yield int(self.off[b]) + i, int(page[i]), int(r[i]), bool(ok[i])


SHAPES = [(128, 28, 4, 16), (64, 14, 2, 7), (32, 8, 8, 24), (16, 6, 1, 1), (128, 5, 5, 64)]
SEQS = [([1], [41]), ([1], [1]), ([3, 0, 20, 1], [3, 5, 900, 16]), ([1700, 4], [1703, 70])]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", SHAPES)
@pytest.mark.parametrize("news,lengths", SEQS, ids=["one", "first", "mixed", "many"])
def test_rows_that_are_not_rotated_are_held_bit_for_bit(D, hq, hkv, R, dtype, news, lengths):
    c = Written(D + R + len(news), news, lengths, D, hq, hkv, R, dtype, order="page_row_head" if R == 16 else "page_head_row")
    was = c.before()
    q = c.cache.append(1, i32(c.table), i32(lengths), c.k, c.v, q=c.q, offsets=i32(c.off))
    assert torch.equal(q, c.q)
    for x, pages, scales, old, old_s in ((c.k, c.kp, c.ks, was[0], was[2]), (c.v, c.vp, c.vs, was[1], was[3])):
        want, e = held(f64(x))
        got, got_e = codes(pages), scales.view(torch.uint8).cpu().numpy().astype(int) - 127
        touched = np.zeros(pages.shape[:4], bool)
        for t, page, r, ok in c.rows():
            assert ok
            assert np.array_equal(got[1, page, :, r], want[t]) and np.array_equal(got_e[1, page, :, r], e[t]), t
            touched[1, page, :, r] = True
        other = torch.tensor(~touched, device="cuda")
        assert torch.equal(pages.view(torch.uint8)[other], old[other]) and torch.equal(scales.view(torch.uint8)[other], old_s[other])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("D,n_rot,axes", [(128, 128, 3), (128, 64, 2), (64, 48, 1), (32, 16, 3), (16, 16, 5), (128, 112, 3)])
def test_rotated_rows(D, n_rot, axes, pairing, dtype):
    news, lengths = [5, 900, 1], [30, 905, 1]
    c = Written(D + n_rot, news, lengths, D, 6, 2, 16, dtype)
    rng = c.rng
    inv = 1e4 ** (-2.0 * np.arange(n_rot // 2) / n_rot)
    axis = rng.integers(0, axes, n_rot // 2).astype(np.int32)
    pos = rng.integers(0, 300000, (axes, c.T)).astype(np.int32)
    rope = mk.Rope(torch.tensor(inv, device="cuda"), i32(axis), n_axes=axes, pairing=pairing)
    out = c.q if n_rot == 48 else None                          # in place, too
    given = f64(c.q)
    q = c.cache.append(0, i32(c.table), i32(lengths), c.k, c.v, q=c.q, offsets=i32(c.off), rope=rope, positions=i32(pos), q_out=out)
    near(f64(q), rotated(given, pos, inv, axis, pairing), rotation_error(given, n_rot, pairing, far=3e5), dtype)
    k = f64(c.k)
    want, err = rotated(k, pos, inv, axis, pairing), rotation_error(k, n_rot, pairing, far=3e5)
    got, e = stands_for(c.kp, c.ks), c.ks.view(torch.uint8).cpu().numpy().astype(int) - 127
    vw, ve = held(f64(c.v))
    for t, page, r, ok in c.rows():
        x, f, g = want[t], e[0, page, :, r], got[0, page, :, r]
        # half a step: 2^-4 of the value, or 2^(e-10) below 2^(e-6)
        tol = err[t] + np.maximum(2.0**-4 * (np.abs(x) + err[t]), np.ldexp(1.0, f - 10)[:, None])
        assert (np.abs(g - x) <= tol).all(), t
        most, by = np.abs(x).max(-1), err[t].max(-1)
        assert (most - by <= np.ldexp(448.0, f)).all() and (most + by > np.ldexp(448.0, f - 1)).all(), t
        assert np.array_equal(codes(c.vp[0, page, :, r]), vw[t])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_features_at_the_edges_of_the_form(dtype):
    D = 64
    x = np.zeros((14, 1, D))
    x[1, 0, 3] = np.inf
    x[2, 0] = np.nan
    x[3, 0, :] = 2.0 ** -np.arange(D)                       # down to codes of zero
    x[4, 0, 0], x[4, 0, 1:] = 448.0, 448.0 * 2.0**-15 * np.linspace(0.0, 4.0, D - 1)   # steps of 2^-9, their ties among them
    x[5, 0, :3] = 1.75, -np.inf, 1e-3                       # the largest as large as its exponent allows
    x[6, 0, :2] = 1.7578125, np.nan                         # the next bf16 number
    x[7, 0, :3] = 3.3e38, -3.3e38, 2.6e38                   # past 448 * 2^119
    x[8, 0, :3] = 1e-38, -3e-39, 0.0                        # below every exponent
    x[9, 0] = -0.0
    x[10, 0] = np.arange(D) / 16 + 15                       # ties of 4 bits
    x[11, 0] = -(np.arange(D) / 16 + 15)
    x[12, 0, 5] = -1e-30
    x[13, 0] = np.where(np.arange(D) % 2, 1e38, -1e-38)
    k = torch.tensor(x, dtype=torch.float32).to(dtype).cuda()
    v = k.flip(-1)
    kp, vp, ks, vs = random_cache(np.random.default_rng(1), (1, 2, 1, 8, D))
    cache = mk.PagedKV8(kp, vp, ks.view(torch.uint8), vs.view(torch.uint8), n_q_heads=1, dtype=dtype)
    table, lengths, off = i32([[1, 0]]), i32([14]), i32([0, 14])
    cache.append(0, table, lengths, k, v.contiguous(), offsets=off)
    back = cache.read(0, table, lengths, off, n_tokens=14)
    for given, pages, scales, got in ((k, kp, ks, back[0]), (v, vp, vs, back[1])):
        want, e = held(f64(given))
        at = [1] * 8 + [0] * 6, list(range(8)) + list(range(6))
        have = codes(pages)[0, at[0], 0, at[1]]
        assert np.array_equal(have, want[:, 0], equal_nan=True)
        assert np.array_equal(scales.view(torch.uint8).cpu().numpy()[0, at[0], 0, at[1]].astype(int) - 127, e[:, 0])
        assert np.array_equal(f64(got)[:, 0], np.ldexp(want, e[..., None])[:, 0], equal_nan=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,hq,hkv,R", SHAPES)
@pytest.mark.parametrize("order", ["page_head_row", "page_row_head", "head_page_row"])
def test_rows_come_back_as_they_stand(D, hq, hkv, R, dtype, order):
    lengths = [1, 333, 0, 64, 7, 2100]
    rng = np.random.default_rng(D + R)
    table, n_pages = spread_tables(rng, lengths, R)
    pages = random_cache(rng, (2, n_pages, hkv, R, D), order=order, slack=16 if order == "page_head_row" else 0)
    cache = mk.PagedKV8(*pages, n_q_heads=hq, dtype=dtype)
    k, v = stands_for(pages[0], pages[2]), stands_for(pages[1], pages[3])
    news = [1, 333, 0, 3, 9, 2100]                              # the fifth asks for rows before its first one: zeros
    off = np.concatenate([[0], np.cumsum(news)])
    table[5, 1] = -1 if R < 64 else table[5, 1]                 # a page that does not exist: zeros
    T = int(off[-1])
    got = cache.read(1, i32(table), i32(lengths), i32(off), n_tokens=T + 5)
    for x, values in zip(got, (k, v)):
        want = np.zeros((T + 5, hkv, D))
        for b, n in enumerate(news):
            page, r, ok = places(table, lengths, R, n_pages, b, np.arange(lengths[b] - n, lengths[b]))
            want[off[b]:off[b + 1]][ok] = values[1][page, :, r][ok]
        assert np.array_equal(f64(x), want)
    out = torch.full((hkv, T, D + 8), 9.0, dtype=dtype, device="cuda")
    kv = [out.clone()[..., :D].transpose(0, 1) for _ in "kv"]
    same = cache.read(1, i32(table), i32(lengths), i32(off), k_out=kv[0], v_out=kv[1])
    assert all(torch.equal(x, y[:T]) for x, y in zip(same, got))
    assert (kv[0]._base[..., D:] == 9.0).all()


def test_rows_without_a_place_are_dropped():
    c = Written(5, [4, 6, 3], [2, 20, 9], 64, 4, 2, 8, BF16)    # the first's first two tokens would be rows -2 and -1
    c.table[1, 1] = 10**6
    c.table[2, 0], c.table[2, 1] = -7, c.table[2, 1]
    was = c.before()
    c.cache.append(0, i32(c.table), i32(c.lengths), c.k, c.v, offsets=i32(c.off))
    written = {(p, r) for _, p, r, ok in c.rows() if ok}
    changed = (c.kp.view(torch.uint8) != was[0]).any(-1)[0].any(1).cpu().numpy()
    assert {tuple(x) for x in np.argwhere(changed)} <= written and len(written) == 2 + 4 + 1
    want, _ = held(f64(c.k))
    for t, page, r, ok in c.rows():
        if ok:
            assert np.array_equal(codes(c.kp[0, page, :, r]), want[t])


def test_offsets_far_past_32_bits():
    """Rows whose pages and scales lie past 4 GiB."""
    D, R, n = 128, 1024, 34000
    kp = torch.zeros(1, n, 1, R, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    vp = torch.zeros(1, n, 1, R, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    big = torch.zeros(n, 130 * 1024, dtype=torch.uint8, device="cuda")   # a page's scales 130 KiB apart
    ks = big.as_strided((1, n, 1, R), (0, 130 * 1024, 0, 1))
    vs = big.as_strided((1, n, 1, R), (0, 130 * 1024, 0, 1), storage_offset=2048)
    cache = mk.PagedKV8(kp, vp, ks, vs, n_q_heads=2)
    table, lengths, off = i32([[n - 1, 3, n - 2]]), i32([2500]), i32([0, 1500])
    k = torch.randn(1500, 1, D, device="cuda").bfloat16()
    v = torch.randn(1500, 1, D, device="cuda").bfloat16()
    cache.append(0, table, lengths, k, v, offsets=off)
    a, b = cache.read(0, table, lengths, off, n_tokens=1500)
    for x, y in ((k, a), (v, b)):
        c, e = held(f64(x))
        assert np.array_equal(f64(y), np.ldexp(c, e[..., None]))


def test_captured_and_replayed():
    c = Written(9, [1] * 5, [17, 3, 900, 63, 1], 128, 8, 2, 16, BF16)
    table, lengths = i32(c.table), i32(c.lengths)
    graph = torch.cuda.CUDAGraph()
    c.cache.append(0, table, lengths, c.k, c.v)
    outs = c.cache.read(0, table, lengths, None, n_tokens=5)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.cache.append(0, table, lengths, c.k, c.v)
        c.cache.read(0, table, lengths, None, k_out=outs[0], v_out=outs[1])
    for i in range(4):
        c.qkv.normal_()
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        w, e = held(f64(c.k))
        assert np.array_equal(f64(outs[0]), np.ldexp(w, e[..., None]))
        lengths += 1 if i == 0 else 0                          # (rows move on: nothing about them is kept on the host)
        lengths.clamp_(max=int(table.shape[1]) * 16)
