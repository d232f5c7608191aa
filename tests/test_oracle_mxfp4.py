"""The oracle's MXFP4 rounding against brute force: every code of every admissible exponent, over values at, next to
and between the borders."""
import numpy as np

from oracle.numerics import E2M1_VALUES, mxfp4_blocks, round_mxfp4_rows


def _brute(block):
    top = max(abs(v) for v in block)
    e = -100
    while e < 125 and top > 7 * 2.0 ** e:
        e += 1
    out = []
    for v in block:
        y = abs(v) / 2.0 ** e
        best = min(range(8), key=lambda c: (abs(E2M1_VALUES[c] - y), c % 2))
        out.append(np.copysign(E2M1_VALUES[best] * 2.0 ** e, v))
    return out


def test_values_around_every_border():
    rng = np.random.default_rng(0)
    mid = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0]
    near = sorted({s * m * (1 + d) for m in mid + list(E2M1_VALUES) for d in (0, 2.0 ** -23, -(2.0 ** -23), 0.1) for s in (1, -1)})
    for e in (-101, -100, -99, -20, 0, 1, 30, 124, 125, 126):
        for top in (4.0, 5.9, 6.0, 7.0, 7.0 * (1 + 2.0 ** -23)):
            x = rng.choice(near, 31)
            block = np.append(np.clip(x, -top, top), top) * 2.0 ** e
            assert np.array_equal(round_mxfp4_rows(block), _brute(block)), (e, top)


def test_no_value_is_off_by_more_than_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2000, 64)) * np.exp(4 * rng.standard_normal((2000, 1)))
    codes, e = mxfp4_blocks(x)
    assert codes.shape == x.shape and e.shape == (2000, 2)
    y = np.abs(x).reshape(2000, 2, 32) / np.exp2(e)[..., None]
    assert y.max() <= 7 and (y.max(-1) > 3.5).all()
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    got = np.abs(round_mxfp4_rows(x)).reshape(2000, 2, 32) / np.exp2(e)[..., None]
    assert (np.abs(got - y) <= step / 2).all()
    # rounded again, nothing moves
    assert np.array_equal(round_mxfp4_rows(round_mxfp4_rows(x)), round_mxfp4_rows(x))


def test_zeros_and_values_without_a_number():
    x = np.zeros((5, 64))
    x[1, 3], x[2, 40], x[3, 7] = np.nan, np.inf, 2.0 ** -103
    got = round_mxfp4_rows(x)
    assert np.isnan(got[1, :32]).all() and not got[1, 32:].any()
    assert np.isnan(got[2, 32:]).all() and not got[2, :32].any()
    assert not got[[0, 3, 4]].any()
