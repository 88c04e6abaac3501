"""8-bit pages at the ends of the numbers' range: rows whose powers of two lie far apart,
and the largest numbers of bf16. Tolerances as in test_gpu_paged."""

import numpy as np
import pytest
import torch

from gpu_cases import ensure_lib, f64
from oracle import paged as opaged
from test_gpu_paged import Pages, check_decode, ints, randn, sums

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,lens", [(8, 2, [300, 5000]), (2, 2, [40, 700]), (16, 1, [900, 30]), (32, 8, [6000, 1, 9000, 77])])
@pytest.mark.parametrize("order", ["mixed", "small first", "large first"])
def test_values_of_far_apart_sizes(d, hq, hkv, lens, order):
    """Half of the V rows are zeros (power -80) and half 2^70: a zero row adds nothing to the
    numerator, but its weight counts in the sum of weights as any other's."""
    p = Pages(lens, hq, hkv, d, 32, "e4m3", [0] * hkv)
    k, v = randn((sum(lens), hkv, d), 1), randn((sum(lens), hkv, d), 2)
    v *= 2.0 ** 70
    at = sums(lens)
    for a, n in zip(at, lens):
        if order == "mixed":
            v[a:a + n:2] = 0
        elif order == "small first":
            v[a:a + (n + 1) // 2] = 0
        else:
            v[a + n // 2:a + n] = 0
    p.cache.append(k, v, ints(lens), p.table, cu_rows=ints(at))
    q = randn((len(lens), hq, d), 3)
    held = [(p.held(f64(k[a:b])), p.held(f64(v[a:b]))) for a, b in zip(at, at[1:])]
    for max_len in (0, 100):
        out = torch.full_like(q, float("nan"))
        p.cache.decode(q, ints(lens), p.table, out, max_len=max_len)
        p.cache.check()
        check_decode(out, q, held, [0] * hkv, 0, 1, f"{order} {max_len}")


@pytest.mark.parametrize("d", [64, 128])
def test_a_finite_number_stays_finite(d):
    """The largest numbers: with a power of 120 a code of 256 or more would stand for more than
    bf16 holds."""
    hkv, page = 2, 16
    most = torch.finfo(torch.bfloat16).max
    x = randn((20, hkv, d), 1)
    for i, big in enumerate((most, -most, 1.9375 * 2.0 ** 127, 1.8828125 * 2.0 ** 127, 1.875 * 2.0 ** 127, -2.0 ** 127)):
        x[i, 0, 5] = big
    x[7, 1, 3], x[7, 1, 4], x[8, 0, 0], x[8, 0, 1] = most, float("inf"), -most, float("nan")
    p = Pages([20], hkv, hkv, d, page, "e4m3", [0] * hkv)
    p.cache.append(x, x, ints([20]), p.table, cu_rows=ints([0, 20]))
    k_out, v_out = torch.empty_like(x), torch.empty_like(x)
    p.cache.read(p.table, ints([0, 20]), k_out, v_out)
    p.cache.check()
    assert torch.equal(torch.isfinite(k_out), torch.isfinite(x)) and torch.equal(k_out.isnan(), v_out.isnan())
    want = opaged.decode(*opaged.encode(f64(x)))
    for out in (k_out, v_out):
        assert np.array_equal(f64(out), want, equal_nan=True)
    err = np.abs(want - f64(x))[np.isfinite(f64(x))]
    size = np.abs(f64(x)).max(-1, where=np.isfinite(f64(x)), initial=0)[..., None].repeat(d, -1)[np.isfinite(f64(x))]
    assert (err <= 2.0 ** -4 * size).all()
