"""8-bit pages at the ends of the numbers' range: rows whose powers of two lie far apart.
Tolerances as in test_gpu_paged."""

import pytest
import torch

from gpu_cases import ensure_lib, f64
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
