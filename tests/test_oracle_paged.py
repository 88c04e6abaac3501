"""The 64-bit definitions of the paged operators against direct sums and torch's own
8-bit type."""

import numpy as np
import pytest
import torch

from oracle import attention as oatt
from oracle import paged


def test_codes_are_the_8_bit_type():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    v = paged.e4m3_values()
    assert np.array_equal(np.isnan(t), np.isnan(v))
    assert np.array_equal(t[~np.isnan(t)], v[~np.isnan(v)])


def test_encode_rounds_to_nearest_even():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 64)) * 2.0 ** rng.integers(-60, 60, (500, 1))
    x[0] = 0
    x[1, :4] = [448, 464, -17, 2.0 ** -10]
    x[2, 0] = 449
    x = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    codes, e = paged.encode(x)
    most = np.abs(x).max(-1)
    y = x / 2.0 ** e[:, None].astype(float)
    assert (np.abs(y) <= 448).all()
    assert ((np.abs(x).max(-1) > 448 * 2.0 ** (e.astype(float) - 1)) | (e == paged.E_MIN)).all()
    t = torch.from_numpy(y).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes, t)
    assert most.shape == e.shape


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_encode_of_a_number_that_is_none(value):
    x = np.full(64, 3.0)
    x[5] = value
    codes, e = paged.encode(x)
    assert codes[5] & 127 == 127
    keep = np.arange(64) != 5
    assert (paged.decode(codes, e)[keep] == 3.0).all()


def test_attend_is_the_prefill_definition():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((40, 4, 8)), rng.standard_normal((40, 2, 8)), rng.standard_normal((40, 2, 8))
    want = oatt.prefill(q, k, v, [0, 1], 3, 7)
    assert np.allclose(paged.attend(q, k, v, [0, 1], 3, 7), want, rtol=1e-12, atol=1e-12)
    assert np.allclose(paged.attend(q[29:], k, v, [0, 1], 3, 7), want[29:], rtol=1e-12, atol=1e-12)


def test_rows_before_the_first_key():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((3, 1, 8)), rng.standard_normal((3, 1, 8))
    out = paged.attend(q, k, v, [0], 0, 1)
    assert (out[:2] == 0).all()
    assert np.allclose(out[2], v[0])
    assert (paged.attend(q, k[:0], v[:0], [1], 2, 4) == 0).all()
