"""Pins of the rows' oracle: the 8-bit numbers against torch's, the rotation against complex products and its own properties."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as R


def test_the_256_numbers_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = R.e4m3_values()
    assert (np.isnan(got) == np.isnan(want)).all() and (got[~np.isnan(got)] == want[~np.isnan(want)]).all()


def test_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal((50, 64)) * 10.0 ** np.random.default_rng(1).uniform(-8, 8, (50, 1))
    x = x.astype(np.float32).astype(np.float64)
    got, e = R.hold(x)
    power = 2.0 ** (e - 127.0)[:, None]
    want = torch.tensor(x / power, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy() * power
    assert (got == want).all()
    top = np.abs(x).max(-1)
    assert (top <= 448 * power[:, 0]).all() and (top > 224 * power[:, 0]).all()
    assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * power)).all()


@pytest.mark.parametrize("x,e", [(0.0, 67), (448.0, 127), (448.0000001, 128), (224.0, 126), (1e-30, 67), (3.3e38, 247), (448 * 2.0 ** -60, 67), (449 * 2.0 ** -60, 68)])
def test_exponents(x, e):
    assert R.hold(np.array([[x, 0.0]]))[1][0] == e


def test_what_is_not_finite_becomes_nan_and_has_no_say():
    v, e = R.hold(np.array([[1.0, np.inf, -np.inf, np.nan]]))
    assert v[0, 0] == 1.0 and np.isnan(v[0, 1:]).all() and e[0] == R.hold(np.array([[1.0]]))[1][0]


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_is_a_complex_product(neighbours):
    rng = np.random.default_rng(2)
    x, freq = rng.standard_normal((3, 64)), 10000.0 ** (-np.arange(16) / 16)
    y = R.rotate(x, None, 1e-6, 1234, freq, neighbours)
    a = x[:, 0:32:2] + 1j * x[:, 1:32:2] if neighbours else x[:, :16] + 1j * x[:, 16:32]
    b = y[:, 0:32:2] + 1j * y[:, 1:32:2] if neighbours else y[:, :16] + 1j * y[:, 16:32]
    assert np.abs(b - a * np.exp(1j * 1234 * freq)).max() < 1e-12
    assert (y[:, 32:] == x[:, 32:]).all()
    assert np.abs(R.rotate(y, None, 1e-6, -1234, freq, neighbours) - x).max() < 1e-12
    # products of rotated rows depend on the distance of their positions alone
    k = rng.standard_normal((3, 64))
    near, far = ((R.rotate(x, None, 1, p, freq, neighbours) * R.rotate(k, None, 1, p - 7, freq, neighbours)).sum(-1) for p in (7, 5007))
    assert np.abs(near - far).max() < 1e-9


def test_norm():
    x = np.random.default_rng(3).standard_normal((2, 64)) * 5
    y = R.rotate(x, np.full(64, 2.0), 1e-6, 0, np.zeros(0), False)
    assert np.abs((y * y).mean(-1) - 4).max() < 1e-5
