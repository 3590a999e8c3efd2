"""The smoothed loss of rows whose values are large beside their spread, and of spreads beyond the type's range, on the GPU against
the formula in 64 bits, with every difference from the maximum taken first (a mean of the values themselves loses these rows in 64 bits too).

Tolerance.  u = 2^-24.  lse - x_y as in test_cross_entropy_parity.py: rel(s) <= (3 R + 4 + C) u with C = V / 64 + 64, R the row's spread (an
exponential of less than -110 is 0 either way), and four roundings of log s and m - x_y.  m - mean is a sum of terms that are not negative: each is
off by a rounding of the difference, one of 1 / V, one of the product, and the chain has C additions and at most 12 roundings where maxima are joined, so it is off
by (C + 16) u of itself.  Four more roundings join them."""
import numpy as np
import pytest

from paper_2111_04007_amd.synth import to_f64
from tests.test_cross_entropy_parity import U, call

pytestmark = pytest.mark.gpu


def parts(x, y):
    """(log of the sum, how far the target and the mean lie below the maximum)"""
    below = x.max(axis=1, keepdims=True) - x
    return np.log(np.exp(-below).sum(axis=1)), below[np.arange(len(y)), y], below.mean(axis=1)


def bound(x, y, ref, e):
    rows, vocab = x.shape
    top, c = x.max(axis=1), vocab / 64 + 64
    R = np.minimum(top - x.min(axis=1), 110.0)
    gap, lag = parts(x, y)[1:]
    return (3 * R + 4 + c) * U + 4 * U * (2 * np.log(vocab) + 2 * gap) + e * (c + 16) * U * lag + 4 * U * np.abs(ref)


def check(x, y, dtype, vocab, e, lead=0):
    loss, out2, grad, xr = call(x, y, dtype, "i64", vocab, vocab, lead, lead, e)
    e = float(np.float32(e))
    log, gap, lag = parts(xr, y)
    ref = (1 - e) * (log + gap) + e * (log + lag)
    tol = bound(xr, y, ref, e)
    err = np.abs(to_f64(loss) - ref)
    assert (err <= tol).all(), (err / tol).tolist()
    assert abs(float(out2[0]) - ref.sum()) <= tol.sum() + U * abs(ref.sum())
    alone = call(x, y, dtype, "i64", vocab, vocab, lead, lead, e, grad=False)
    assert (alone[0] == loss).all()


@pytest.mark.parametrize("e", [0.1, 1.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,lead", [(1, 0), (2, 1), (13, 0), (2050, 0), (2051, 3), (9001, 0), (30523, 0), (140001, 1), (280001, 0)])
def test_values_large_beside_their_spread(dtype, vocab, lead, e):
    r = np.random.default_rng((vocab, lead))
    x = r.standard_normal((8, vocab))
    y = r.integers(0, vocab, 8)
    x[0] += 3.0e4
    x[1] -= 3.0e4
    x[2] = x[2] * 0.01 - 1.0e6
    x[3] = -3.38e38                                 # the type's lowest, nearly, throughout: log V
    x[4] = 3.38e38
    x[5] = np.linspace(-60.0, 60.0, vocab) + 7.0e3   # the maximum moves with every piece that is read
    x[6] = np.linspace(60.0, -60.0, vocab) + 7.0e3
    x[7, vocab // 2] = 40.0                          # and once, late for some threads
    check(x, y, dtype, vocab, e, lead)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [64, 2050, 30523, 280001])
def test_entries_of_the_lowest_value_and_spreads_beyond_the_range(dtype, vocab):
    """The target is the largest entry, whose distance from itself is 0: the loss is finite however far the others are."""
    r = np.random.default_rng(vocab)
    x = r.standard_normal((4, vocab))
    y = r.integers(8, vocab, 4)
    x[0, :3] = -3.38e38
    x[1, 3:7] = -3.38e38
    x[2, :2] = -3.38e38
    x[2, y[2]] = 3.38e38                             # 6.8e38 apart
    x[3] = 1.0e38
    x[3, ::3] = -3.0e38
    y[3] -= y[3] % 3 == 0
    check(x, y, dtype, vocab, 0.25)
