"""Plain 64-bit forms of the paged cache's operators, and caches to try them on.  A cache of the tests is described by numpy
arrays on the host: pages [layer][page][KV head][row][feature] in float64 (the payload's values exactly), a table, lengths and
offsets; the device's copy of the pages lies in any of three orders of dimensions, with slack between the rows on request."""
import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}  # a rounding to the type, relative to the value


def f64(t):
    return t.detach().double().cpu().numpy()


def on_device(pages, dtype, order="page_head_row", slack=0):
    """[L][page][head][row][D] values as a device tensor of that logical shape, laid out in `order`."""
    t = torch.as_tensor(pages).to(dtype).cuda()
    perm = {"page_head_row": (0, 1, 2, 3, 4), "page_row_head": (0, 1, 3, 2, 4), "head_page_row": (0, 2, 1, 3, 4)}[order]
    back = [perm.index(i) for i in range(5)]
    x = t.permute(perm)
    buf = torch.full((*x.shape[:4], x.shape[4] + slack), 7.0, dtype=dtype, device="cuda")
    buf[..., : x.shape[4]] = x
    return buf[..., : x.shape[4]].permute(back)


def spread_tables(rng, lengths, R, width=None, n_spare=3):
    """A table of shuffled pages for these lengths, -1 past the last; how many pages there are."""
    need = [-(-int(n) // R) for n in lengths]
    width = width or max(max(need), 1)
    n_pages = sum(need) + n_spare
    order = rng.permutation(n_pages)
    table = np.full((len(lengths), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def places(table, lengths, R, n_pages, b, rows):
    """(page, row in it, is there) of the rows of sequence b."""
    rows = np.asarray(rows)
    ok = (rows >= 0) & (rows < table.shape[1] * R)
    page = np.where(ok, table[b][np.where(ok, rows // R, 0)], -1)
    ok = ok & (page >= 0) & (page < n_pages)
    return np.where(ok, page, 0), np.where(ok, rows % R, 0), ok


def rotated(x, positions, inv_freq, axis, pairing, inverse=False):
    """x [T][H][D] in float64; positions [axes][T]."""
    T, _, D = x.shape
    n = 2 * len(inv_freq)
    ax = np.zeros(n // 2, int) if axis is None else axis
    pos = np.stack([positions[a] if 0 <= a < len(positions) else np.zeros(T) for a in ax], -1)
    ang = pos.astype(np.float64) * np.asarray(inv_freq, np.float64) * (-1 if inverse else 1)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = x.copy()
    a, b = (slice(0, n // 2), slice(n // 2, n)) if pairing == "halves" else (slice(0, n, 2), slice(1, n, 2))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rotation_error(x, n, pairing, far=0.0):
    """What a rotated value may be off before its last rounding: the turn is exact to 2^-22 (one conversion, cosine and sine of two
    half steps or so) and, at the largest angle `far`, to the three roundings in 64 bits of both forms; each product and the sum
    round once in fp32."""
    a, b = (slice(0, n // 2), slice(n // 2, n)) if pairing == "halves" else (slice(0, n, 2), slice(1, n, 2))
    e = np.zeros_like(x)
    both = np.abs(x[..., a]) + np.abs(x[..., b])
    e[..., a] = e[..., b] = both * (2.0**-21 + far * 2.0**-51)
    return e


def near(got, want, err, dtype, rounded=True):
    """|got - want| within err and, where the output was rounded to `dtype`, its half step."""
    h = HALF_STEP[dtype] if rounded else 0.0
    tol = err + h * (np.abs(want) + err) + 1e-40
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:5], want[bad][:5], tol[bad][:5] if np.ndim(tol) else tol)


def gathered(pages, layer, table, lengths, R, b, n):
    """Rows 0..n-1 of sequence b as [n][head][D], and which of them are there."""
    page, r, ok = places(table, lengths, R, pages.shape[1], b, np.arange(n))
    return pages[layer][page, :, r], ok


def attention(q, rows_of, lengths, offsets, hkv, causal, room):
    """q [T][Hq][D]; rows_of(b, n) -> k, v [n][Hkv][D] and which rows are there.  Returns out, the weights every row received
    [B][Hkv][n], and for each output the mean of |v| under its weights and the largest sum |q_i k_i| of the rows it sees."""
    T, Hq, D = q.shape
    G = Hq // hkv
    out, amean, reach = np.zeros_like(q), np.zeros_like(q), np.zeros((T, Hq, 1))
    received = []
    for b in range(len(lengths)):
        lo, hi = offsets[b], offsets[b + 1]
        n = min(max(int(lengths[b]), 0), room)
        k, v, there = rows_of(b, n)
        got = np.zeros((hkv, n))
        for i in range(hi - lo):
            seen = there & (np.arange(n) <= max(int(lengths[b]), 0) - (hi - lo) + i) if causal else there
            if not seen.any():
                continue
            for h in range(Hq):
                kk, vv = k[seen, h // G], v[seen, h // G]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = kk @ q[lo + i, h] / np.sqrt(D)
                    w = np.exp(s - s.max())
                    w = w / w.sum()
                    out[lo + i, h] = w @ vv
                    amean[lo + i, h] = w @ np.abs(vv)
                    reach[lo + i, h] = (np.abs(kk) @ np.abs(q[lo + i, h])).max()
                got[h // G, seen] += w
        received.append(got)
    return out, received, amean, reach


def attention_error(amean, reach, n, D, dtype, single_weights=False):
    """What an output may be off before its last rounding.  A score: its products add up in fp32 (bf16 payloads: D terms in an order of
    the matrix core's; fp32: sums of four joined pair by pair), a weight is off by that and the exponential's own two steps, in numerator and
    denominator; sums over n rows, 16 at a time and more; bf16 payloads: the weight as a pair of bf16 (2^-16), or as one (2^-8), in numerator
    and denominator."""
    terms = D if dtype == torch.bfloat16 else 12
    score = (terms + 4) * 2.0**-24 * reach / np.sqrt(D)
    rel = 2 * score + (n / 16 + 20) * 2.0**-24
    if dtype == torch.bfloat16:
        rel = rel + (2.0**-7 if single_weights else 2.0**-16)
    return amean * rel
