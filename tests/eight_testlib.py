"""Rows in 8 bits by their definition, in 64 bits on the host, and caches of them to try operators on."""
import numpy as np
import torch

LEAST, MOST = -117, 119   # exponents of a row's power of two


def e4m3(x):
    """The nearest e4m3 number, ties to the even one; at most 448, NaN where x is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    mag = np.where(fine, np.minimum(np.abs(x), 448.0), 0.0)
    _, e = np.frexp(np.where(mag > 0, mag, 1.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(fine, np.copysign(np.rint(mag / step) * step, x), np.nan)


def exponents(x):
    """Of rows [..., feature]: the smallest e with max |x| <= 448 * 2^e over the finite features, inside LEAST .. MOST."""
    x = np.asarray(x, np.float64)
    most = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    m, e = np.frexp(most)             # most = m * 2^e, m in 1/2 .. 1; 448 = 7/8 * 2^9
    return np.clip(np.where(most > 0, e - 9 + (m > 0.875), LEAST), LEAST, MOST).astype(np.int64)


def held(x):
    """(codes' values, exponents) of rows."""
    x = np.asarray(x, np.float64)
    e = exponents(x)
    return e4m3(np.ldexp(x, -e[..., None])), e


def codes(t):
    """What float8_e4m3fn numbers on the device stand for."""
    b = t.view(torch.uint8).cpu().numpy().astype(np.int64)
    s, e, m = b >> 7, b >> 3 & 15, b & 7
    v = np.where(e > 0, np.ldexp(1.0 + m / 8.0, e - 7), np.ldexp(m / 8.0, -6))
    return np.where((b & 127) == 127, np.nan, np.where(s == 1, -v, v))


def stands_for(pages, scales):
    """The rows of pages and scales in 64 bits."""
    return np.ldexp(codes(pages), scales.view(torch.uint8).cpu().numpy().astype(np.int64)[..., None] - 127)


ORDERS = {"page_head_row": (0, 1, 2, 3), "page_row_head": (0, 1, 3, 2), "head_page_row": (0, 2, 1, 3)}


def laid_out(t, order, slack=0):
    """A tensor [layer][page][head][row](, [feature]) of the same values on the device, in another order of memory."""
    perm = list(ORDERS[order]) + ([4] if t.dim() == 5 else [])
    x = t.permute(perm)
    buf = torch.full((*x.shape[:-1], x.shape[-1] + slack), 0x55, dtype=torch.uint8, device="cuda")
    buf[..., : x.shape[-1]] = x.view(torch.uint8).cuda()
    return buf[..., : x.shape[-1]].permute([perm.index(i) for i in range(t.dim())]).view(t.dtype)


def random_cache(rng, shape, spread=2, order="page_head_row", slack=0):
    """k_pages, v_pages, k_scales, v_scales of random rows [layer][page][head][row][feature]: normal numbers of several sizes."""
    got = []
    for _ in "kv":
        c, e = held(rng.standard_normal(shape) * np.exp2(rng.integers(-spread, spread + 1, shape[:4]))[..., None])
        got.append((torch.tensor(c, dtype=torch.float32).to(torch.float8_e4m3fn), torch.tensor(e + 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)))
    (kp, ks), (vp, vs) = got
    return [laid_out(t, order, slack) for t in (kp, vp)] + [laid_out(t, order) for t in (ks, vs)]
