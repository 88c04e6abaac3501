"""Norms and rotation without a GPU: the frequencies that a rope holds, the 64-bit definition, and
what the binding and the library refuse (before any pointer reaches a kernel)."""

import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh
from paper_2608_06849_gb300 import build as aoh_build
from test_paged_checks import Cuda, bf, cache, ints, refused


@pytest.fixture(scope="module", autouse=True)
def lib():
    aoh_build.build()
    return aoh.load()


def inverse_two_pi():
    """1 / (2 pi) to 200 bits, by Machin's series."""
    def arctan_inv(x):
        s, term, k = Fraction(0), Fraction(1, x), 0
        while term.numerator and abs(term) > Fraction(1, 2 ** 230):
            s += term / (2 * k + 1) * (-1) ** k
            term /= x * x
            k += 1
        return s
    pi = 4 * (4 * arctan_inv(5) - arctan_inv(239))
    return 1 / (2 * pi)


@pytest.mark.parametrize("freqs", [
    [500000.0 ** (-2 * i / 128) for i in range(64)],
    [-1e6 + 31250.7 * i for i in range(64)],
    [math.pi, -math.pi, 2 * math.pi, 1e-12, -1e-12, 0.0, 5e-324, 1.0],
])
def test_turns_are_the_fractions_of_a_turn(freqs):
    """Each entry is the frequency over 2 pi, whole turns dropped, in units of 2^-64: to within
    two units (its two roundings, and that of 1 / (2 pi) to 107 bits times 1e6 / 2 pi < 2^18)."""
    r = aoh.Rope(inv_freq=freqs)
    x = inverse_two_pi()
    for f, t in zip(freqs, r.c.turns):
        off = (Fraction(f) * x * 2 ** 64 - t) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= 2
    assert r.c.n_pairs == len(freqs) and r.c.interleaved == 0 and r.c.scale == 1.0


def test_rope_arguments():
    assert aoh.Rope(64, base=1e4).c.n_pairs == 32
    assert aoh.Rope(0).c.n_pairs == 0
    assert aoh.Rope(inv_freq=[]).c.n_pairs == 0
    assert aoh.Rope(16, interleaved=True, scale=1.5).c.interleaved == 1
    same = aoh.Rope(inv_freq=[1e6 ** (-2.0 * i / 128) for i in range(64)])
    assert list(same.c.turns) == list(aoh.Rope(128, base=1e6).c.turns)
    for bad in (dict(rotated=24), dict(rotated=144), dict(inv_freq=[1.0] * 7),
                dict(inv_freq=[float("nan")] * 8), dict(inv_freq=[2e6] * 8)):
        with pytest.raises(aoh.AohError):
            aoh.Rope(**bad)
    for bad in (dict(), dict(rotated=64, inv_freq=[1.0] * 32), dict(rotated=15), dict(rotated=-16), dict(rotated=64, scale=float("inf")),
                dict(rotated=64, scale=float("nan"))):
        with pytest.raises(ValueError):
            aoh.Rope(**bad)


@pytest.mark.parametrize("base", [0, 0.0, -1e4, float("nan")])
def test_rope_bases_that_have_no_powers(base):
    """A refusal in the binding's own words, not of the arithmetic behind it."""
    with pytest.raises(ValueError, match="above 0"):
        aoh.Rope(64, base=base)


def test_rope_struct_matches_header():
    assert ctypes.sizeof(aoh.aoh_rope) == 16 + 64 * 8
    assert aoh.aoh_rope.turns.offset == 16
    assert ctypes.sizeof(aoh.aoh_norms) == 24


def test_rotation_of_the_definition():
    """Scores depend on the distance of positions alone, and position 0 turns nothing."""
    g = np.random.default_rng(0)
    q, k = g.standard_normal((2, 1, 1, 64))
    f = orot.frequencies(64, 1e4)
    for il in (False, True):
        at = lambda x, p: orot.rotate(x, [p], f, il)  # noqa: E731
        assert np.array_equal(at(q, 0), q)
        assert np.isclose((at(q, 907) * at(k, 900)).sum(), (at(q, 7) * at(k, 0)).sum())
    x = orot.norm(q, np.ones(64), 0.0)
    assert np.isclose((x * x).mean(), 1.0)


def fp(n, dtype=torch.float32):
    return Cuda(torch.ones(n, dtype=dtype))


def test_norm_rotate_tensors():
    rope, f = aoh.Rope(64), aoh.aoh_norm_rotate
    q, k, p = bf(5, 8, 64), bf(5, 2, 64), ints(5)
    refused("q with q_out", f, rope, None, None, p, None, None)
    refused("q with q_out", f, rope, q, k, p, q, None)
    refused("expected \\[rows, heads, d\\]", f, rope, bf(5, 512), k, p, q, k)
    refused("^k has shape", f, rope, q, bf(5, 2, 128), p, q, k)
    refused("^k has shape", f, rope, q, bf(5, 128), p, q, k)
    refused("^q_out has shape", f, rope, q, k, p, bf(5, 4, 64), k)
    refused("^k and k_out hold", f, rope, q, bf(4, 2, 64), p, q, bf(4, 2, 64))
    refused("^positions has shape", f, rope, q, k, ints(4), q, k)
    refused("^positions must be", f, rope, q, k, Cuda(torch.zeros(5, dtype=torch.int64)), q, k)
    refused("bfloat16", f, rope, Cuda(torch.zeros(5, 8, 64)), k, p, q, k)
    refused("^q_norm has shape", f, rope, q, k, p, q, k, q_norm=fp(32))
    refused("^k_norm must be", f, rope, q, k, p, q, k, k_norm=fp(64, torch.float16))
    refused("^q_norm must be", f, rope, q, k, p, q, k, q_norm=torch.ones(64))
    refused("of one type", f, rope, q, k, p, q, k, q_norm=fp(64), k_norm=fp(64, torch.bfloat16))
    refused("dense rows", f, rope, Cuda(torch.zeros(5, 64, 8, dtype=torch.bfloat16).transpose(1, 2)), k, p, q, k)


def test_append_rotated_tensors():
    c, rope = cache(), aoh.Rope(64)
    q, k, lens, table = bf(3, 8, 64), bf(3, 2, 64), ints(3), ints(3, 9)
    f = c.append_rotated
    refused("for 4 sequences", f, rope, q, k, k, ints(4), ints(4, 9), q)
    refused("^q, k, v and q_out hold", f, rope, q, k, bf(2, 2, 64), lens, table, q)
    refused("^q, k, v and q_out hold", f, rope, q, k, k, lens, table, bf(4, 8, 64))
    refused("^q, k, v and q_out hold", f, rope, bf(2, 8, 64), k, k, lens, table, q)
    refused("^q has shape", f, rope, k, k, k, lens, table, q)
    refused("^q_out has shape", f, rope, q, k, k, lens, table, k)
    refused("^lens has shape", f, rope, q, k, k, ints(2), table, q)
    refused("^table must be", f, rope, q, k, k, lens, Cuda(torch.zeros(9, 3, dtype=torch.int32).t()), q)
    refused("^cu_rows has shape", f, rope, q, k, k, lens, table, q, cu_rows=ints(3))
    refused("^positions has shape", f, rope, q, k, k, lens, table, q, positions=ints(4))
    refused("^k_norm has shape", f, rope, q, k, k, lens, table, q, k_norm=fp(128))


def test_library_refuses_on_the_host(lib):
    p = ctypes.c_void_p(1 << 20)
    rope = aoh.Rope(64).c

    def call(rope=rope, q=p, k=p, qs=512, ks=128, qn=None, kind=0, eps=1e-6, pos=p, n=1, hq=8, hkv=2, d=64, qo=p, ko=p,
             qos=512, kos=128):
        norms = aoh.aoh_norms(qn, None, kind, eps)
        return lib.aoh_norm_rotate(rope if rope is None else ctypes.byref(rope), ctypes.byref(norms), q, k, qs, ks, pos, n, hq,
                                   hkv, d, qo, ko, qos, kos, None)

    assert call(n=0) == 0 and call(hq=0, hkv=0) == 0
    assert call(d=96) == 5
    for bad in (dict(rope=None), dict(q=None), dict(q=ctypes.c_void_p((1 << 20) + 8)), dict(qs=511), dict(qs=504),
                dict(ks=120), dict(qs=1 << 31), dict(kos=1 << 31), dict(qn=p, kind=2), dict(qn=p, eps=-1.0), dict(qn=p, eps=float("nan")), dict(pos=None), dict(n=-1),
                dict(hq=-1), dict(hq=1025), dict(ko=None), dict(qos=1024), dict(kos=136), dict(qn=ctypes.c_void_p((1 << 20) + 1)),
                dict(rope=aoh.Rope(128).c)):
        assert call(**bad) == 1, bad
    wrong = aoh.Rope(64).c
    wrong.n_pairs = 7
    assert call(rope=wrong) == 1 and "multiple of 8" in lib.aoh_last_error().decode()
    wrong.n_pairs, wrong.interleaved = 8, 3
    assert call(rope=wrong) == 1
    wrong.interleaved, wrong.scale = 0, float("nan")
    assert call(rope=wrong) == 1
    assert lib.aoh_paged_append_rotated(None, ctypes.byref(rope), None, p, p, p, 512, 128, 128, None, None, p, 1, 1, p, 1, p,
                                        512, None) == 1
    assert lib.aoh_rope_init(None, 0, 0, None) == 1
    assert lib.aoh_rope_init(None, 8, 0, ctypes.byref(wrong)) == 1
    assert lib.aoh_rope_init((ctypes.c_double * 8)(), 8, 2, ctypes.byref(wrong)) == 1


def test_attend_tensors():
    c = cache()
    q, lens, table, out = bf(9, 8, 64), ints(3), ints(3, 9), bf(9, 8, 64)
    f = c.attend
    refused("^q has shape", f, bf(9, 2, 64), [3, 3, 3], lens, table, out)
    refused("^out has shape", f, q, [3, 3, 3], lens, table, bf(8, 8, 64))
    refused("one length for each", f, q, [3, 6], lens, table, out)
    refused("one length for each", f, q, [3, 3, 3], lens, table, out, k_lens=[1])
    refused("q_lens say 8", f, q, [3, 3, 2], lens, table, out)
    refused("^lens has shape", f, q, [3, 3, 3], ints(2), table, out)
    refused("^table has shape", f, bf(5, 8, 64), [1] * 5, ints(5), ints(5, 9), bf(5, 8, 64))
    refused("^table must be", f, q, [3, 3, 3], lens, Cuda(torch.zeros(9, 3, dtype=torch.int32).t()), out)
    refused("contiguous", f, q, [3, 3, 3], lens, table, Cuda(torch.zeros(9, 16, 64, dtype=torch.bfloat16)[:, :8]))


def test_attend_without_a_handle(lib):
    p, one = ctypes.c_void_p(1 << 20), (ctypes.c_int32 * 1)(1)
    assert lib.aoh_paged_attend(None, p, 512, one, p, None, 1, p, 1, p, None) == 1
