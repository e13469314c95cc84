"""The reference of the 4-bit tests against what the format promises."""
import numpy as np

import pack4_plain as K


def rows(seed, n=200):
    g = np.random.Generator(np.random.Philox(key=[seed, 4]))
    x = g.standard_normal((n, 128)) * np.exp2(g.integers(-30, 30, (n, 1)))
    x[:, 32:64] *= np.exp2(g.integers(-12, 12, (n, 32)))
    x[g.random((n, 128)) < 0.05] = 0
    x[3, 64:96] = 0
    return x


def test_errors_are_what_is_promised():
    x = rows(1)
    code, scale = K.encode(x)
    y = K.decode(code, scale)
    s = np.repeat(np.ldexp(1.0, scale.astype(int) - 127), 32, axis=-1)
    off, mag = np.abs(x - y), np.abs(x)
    assert np.all(off <= s)
    assert np.all(off[mag < 4 * s] <= 0.5 * s[mag < 4 * s]) and np.all(off[mag < 2 * s] <= 0.25 * s[mag < 2 * s])
    a = mag.reshape(-1, 4, 32).max(-1)
    assert np.all(s.reshape(-1, 4, 32)[..., 0][a > 0] < a[a > 0] / 3.5)


def test_what_was_read_back_stays():
    code, scale = K.encode(rows(2))
    again = K.encode(K.decode(code, scale))
    assert np.array_equal(again[0], code) and np.array_equal(again[1], scale)


def test_ties_edges_and_not_numbers():
    x = np.zeros((6, 128))
    x[0, :14] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -7]
    x[1, 0], x[1, 32], x[1, 64] = 7.0000001, 3.4e38, 2.0 ** -140
    x[2, 5], x[2, 40], x[2, 70] = np.nan, np.inf, -np.inf
    code, scale = K.encode(x)
    y = K.decode(code, scale)
    assert list(y[0, :14]) == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -6]   # (ties to even codes; 7 is 6 at most)
    assert y[1, 0] == 8 and y[1, 32] == 6 * 2.0 ** 125 and y[1, 64] == 0
    assert list(scale[1]) == [128, 252, 3, 3] and list(scale[2]) == [255, 255, 255, 3]
    assert np.isnan(y[2, :96]).all() and (y[2, 96:] == 0).all()
