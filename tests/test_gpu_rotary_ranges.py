"""Norms over the whole range of rows that have one (include/aoh.h), against the 64-bit definition (oracle.rotary).

Tolerance: as in test_gpu_rotary.py (bf16's rounding and 2^-20 of the numbers that make up an output), and where an
output is below bf16's normal numbers half a step of those, 2^-134; 2^-133 is allowed."""

import numpy as np
import pytest
import torch

from gpu_cases import ensure_lib, f64
from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh
from test_gpu_rotary import definition, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


def rows(n, heads, d, low, high, seed):
    """A row's numbers around 2^e, e from low to high over the rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g, device="cuda").clamp(-3.5, 3.5)
    e = torch.linspace(low, high, n, device="cuda").round().view(n, 1, 1)
    # (in two steps: 2^-130 is no normal number)
    return (x * torch.exp2(torch.div(e, 2, rounding_mode="floor")) * torch.exp2(torch.div(e + 1, 2, rounding_mode="floor"))).bfloat16()


@pytest.mark.parametrize("eps, low", [(0.0, -59), (1e-45, -59), (1e-36, -59), (1e-30, -126), (1e-6, -126), (1.0, -126), (1e30, -126)])
@pytest.mark.parametrize("d, rotated, il", [(128, 128, False), (64, 32, True)])
def test_norms_of_any_size(d, rotated, il, eps, low):
    n, hq, hkv = 253, 3, 1
    q, k = rows(n, hq, d, low, 58, 1), rows(n, hkv, d, 58, low, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda"))
    pos = np.arange(n) * 7
    freqs = orot.frequencies(rotated, 1e4)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    aoh.aoh_norm_rotate(aoh.Rope(inv_freq=freqs, interleaved=il), q, k, ints(pos), q_out, k_out, q_norm=w, k_norm=w, eps=eps)
    for x, out in ((q, q_out), (k, k_out)):
        want, size = definition(x, w, float(np.float32(eps)), pos, freqs, il, 1.0)
        off = np.abs(f64(out) - want) - 2.0 ** -8 * np.abs(want) - 2.0 ** -20 * size - 2.0 ** -133
        assert off.max() <= 0, f"row {np.unravel_index(off.argmax(), off.shape)} is {off.max():.3e} beyond the tolerance"


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_norms_of_any_size_on_the_way_into_pages(form):
    """The queries, and the keys as the pages give them back, of rows of 2^-58 and 2^58 are those of the same rows
    times a power of two near one, whose norms are the same."""
    n, hq, hkv, d = 40, 4, 2, 128
    q, k, v = rows(n, hq, d, 0, 0, 1), rows(n, hkv, d, 0, 0, 2), rows(n, hkv, d, 0, 0, 3)
    ones = torch.ones(d, device="cuda")
    got = []
    for e in (0, -58, 58):
        c = aoh.PagedCache(3, 16, hq, hkv, d, 4, 30, [0, 1], form=form, max_seqs=1)
        table, lens, cu = ints([[2, 0, 1]]), ints([n]), ints([0, n])
        out = torch.empty_like(q)
        c.append_rotated(aoh.Rope(d), (q.float() * 2.0 ** e).bfloat16(), (k.float() * 2.0 ** e).bfloat16(), v, lens, table,
                         out, cu_rows=cu, q_norm=ones, k_norm=ones, eps=0.0)
        k_out, v_out = torch.empty_like(k), torch.empty_like(v)
        c.read(table, cu, k_out, v_out)
        c.check()
        got.append((out, k_out, v_out))
    step = 2.0 ** -3 if form == "e4m3" else 2.0 ** -7  # a rounding the other way, to the neighbouring number
    for x in got[1:]:
        for a, b in zip(got[0], x):
            a, b = a.double(), b.double()
            assert torch.isfinite(b).all() and ((a - b).abs() <= step * a.abs().clamp(min=2.0 ** -6)).all()
            assert (a == b).double().mean() > 0.99


def test_rows_of_zeros_and_of_numbers_that_are_not_finite():
    """As the definition: zeros over the root of eps, infinities over themselves NaN and others by them zero."""
    d = 64
    q = torch.zeros((3, 1, d), dtype=torch.bfloat16, device="cuda")
    q[1, 0, 5] = float("inf")
    q[1, 0, 6] = 3.0
    q[2, 0, 7] = float("nan")
    ones, out = torch.ones(d, device="cuda"), torch.empty_like(q)
    aoh.aoh_norm_rotate(aoh.Rope(0), q, None, ints([0, 1, 2]), out, None, q_norm=ones, eps=1e-6)
    assert (out[0] == 0).all() and out[1, 0, 5].isnan() and out[1, 0, 6] == 0 and out[2].isnan().all()
    aoh.aoh_norm_rotate(aoh.Rope(0), q[:1], None, ints([0]), out[:1], None, q_norm=ones, eps=0.0)
    assert out[0].isnan().all()
