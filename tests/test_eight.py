"""The 8-bit form of a row, as the tests reckon it (no GPU here)."""
import numpy as np
import torch

from eight_testlib import codes, e4m3, exponents, held


def test_every_code_is_its_own_nearest():
    b = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn)
    v = codes(b)
    assert np.array_equal(v, b.float().numpy().astype(np.float64), equal_nan=True)
    fine = np.isfinite(v)
    assert np.array_equal(e4m3(v)[fine], v[fine]) and fine.sum() == 254
    up = np.sort(np.unique(v[fine]))
    mid = (up[1:] + up[:-1]) / 2   # ties go to the code whose last bit is 0: the other way from its neighbours
    to = e4m3(mid)
    assert (np.abs(to - mid) == (up[1:] - up[:-1]) / 2).all()
    assert (np.abs(e4m3(mid * (1 + 1e-9)) - mid) <= (up[1:] - up[:-1]) / 2 * (1 + 1e-6)).all()
    x = torch.tensor(np.concatenate([mid, up]), dtype=torch.float32)
    assert np.array_equal(e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).float().numpy().astype(np.float64))


def test_exponents_are_the_smallest():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4000, 16)) * np.exp2(rng.integers(-100, 100, (4000, 1)))
    e = exponents(x)
    most = np.abs(x).max(-1)
    assert (most <= np.ldexp(448.0, e)).all() and (most > np.ldexp(448.0, e - 1)).all()
    edge = np.array([[448.0], [448.0 * (1 + 2.0**-23)], [0.0], [1e-45], [3.4e38], [np.inf], [np.nan]])
    assert exponents(edge).tolist() == [0, 1, -117, -117, 119, -117, -117]
    c, e = held(np.array([[np.inf, 1.0, -np.nan, 3.4e38]]))
    assert np.isnan(c[0, [0, 2]]).all() and c[0, 3] == 448.0 and e[0] == 119
