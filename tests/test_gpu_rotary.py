"""Norms and rotation into dense rows and into pages, against their 64-bit definition
(oracle.rotary; pages: oracle.paged).

Tolerance of a number y of a pair (a, b): stored as bf16 it is off by at most 2^-8 |y|; in 32 bits
the angle is off by at most 2^-25 of a half-turn from the integer's conversion and sincospif by
2 ulp (together under 2^-22), and norm, products and sum by under 12 roundings of 2^-24 each, of
numbers no larger than scale * (|a| + |b|): 2^-20 of that is allowed besides. 8-bit rows: half a step of 3
bits behind the leading one (2^-4 |y|), or of the finest step, 2^-10 * 2^e; the power is the definition's
but where the row's largest number is within 2^-19 of 448 * 2^e."""

import numpy as np
import pytest
import torch

from gpu_cases import ensure_lib, f64
from oracle import paged as opaged
from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


def randn(shape, seed, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    return (x * torch.exp2(spread * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))).bfloat16()


def ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def weights(d, kind, seed):
    if kind is None:
        return None
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(kind)


def definition(x, w, eps, positions, freqs, il, scale):
    """The rotated rows and the size that their tolerance goes by."""
    x = f64(x)
    if w is not None:
        x = orot.norm(x, f64(w), eps)
    y = orot.rotate(x, positions, freqs, il, scale)
    p = len(freqs)
    a, b = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if il else (slice(0, p), slice(p, 2 * p))
    size = np.abs(x)
    size[..., a] = size[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def close(got, want, size, what):
    off = np.abs(f64(got) - want) - 2.0 ** -8 * np.abs(want) - 2.0 ** -20 * size
    assert off.max(initial=-1.0) <= 0, f"{what}: {off.max():.3e} beyond the tolerance at {np.unravel_index(off.argmax(), off.shape)}"


CASES = [
    # rows, Hq, Hkv, d, rotated, interleaved, scale, norms of q and k, fused
    (1, 28, 4, 128, 128, False, 1.0, None, None, False),
    (1, 1, 1, 64, 64, True, 1.0, torch.float32, torch.float32, False),
    (7, 32, 8, 128, 128, False, 1.25, torch.bfloat16, torch.bfloat16, True),
    (33, 8, 2, 64, 32, False, 1.0, torch.float32, None, True),
    (45, 8, 2, 64, 32, True, -0.5, None, torch.bfloat16, False),
    (130, 7, 1, 128, 32, True, 1.0, torch.bfloat16, torch.bfloat16, True),
    (500, 5, 5, 64, 48, False, 1.0, None, None, False),
    (461, 16, 1, 128, 112, False, 2.0, torch.float32, torch.float32, True),
    (1000, 40, 8, 128, 0, False, 3.0, torch.float32, torch.float32, False),
    (2500, 3, 2, 128, 16, True, 1.0, None, torch.float32, False),
    (7400, 12, 4, 64, 64, False, 1.0, torch.bfloat16, torch.bfloat16, True),
]


def inputs(n, hq, hkv, d, fused, seed):
    q, k, v = randn((n, hq, d), seed), randn((n, hkv, d), seed + 1), randn((n, hkv, d), seed + 2)
    if fused:
        # rows that lie on 16 bytes, not on 32
        x = torch.zeros((n, (hq + 2 * hkv) * d + 8), dtype=torch.bfloat16, device="cuda")
        rows = x[:, 8:].unflatten(1, (hq + 2 * hkv, d))
        rows.copy_(torch.cat([q, k, v], 1))
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    return q, k, v


def far_positions(n, seed):
    """From 0 to 2^31 - 1 and some below zero."""
    g = np.random.default_rng(seed)
    p = np.floor(2.0 ** g.uniform(0, 31, n)).astype(np.int64)
    p[::5] *= -1
    p[:1] = 0
    return np.clip(p, -2 ** 31, 2 ** 31 - 1)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_dense(case):
    n, hq, hkv, d, rotated, il, scale, qt, kt, fused = CASES[case]
    q, k, _ = inputs(n, hq, hkv, d, fused, 20 * case)
    pos = far_positions(n, case)
    freqs = orot.frequencies(rotated, 1e4 if case % 2 else 5e5)
    rope = aoh.Rope(inv_freq=freqs, interleaved=il, scale=scale)
    wq, wk = weights(d, qt, 1), weights(d, kt, 2)
    q_out, k_out = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty_like(k, memory_format=torch.contiguous_format)
    aoh.aoh_norm_rotate(rope, q, k, ints(pos), q_out, k_out, q_norm=wq, k_norm=wk, eps=1e-5)
    for x, w, out, what in ((q, wq, q_out, "q"), (k, wk, k_out, "k")):
        want, size = definition(x, w, 1e-5, pos, freqs, il, scale)
        close(out, want, size, f"{what} of case {case}")


def test_one_side_and_in_place():
    n, hq, hkv, d = 77, 8, 2, 128
    q, k, v = inputs(n, hq, hkv, d, True, 3)
    pos, rope = ints(range(5, 5 + n)), aoh.Rope(d)
    q_out, k_out = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda")
    w = weights(d, torch.float32, 0)
    aoh.aoh_norm_rotate(rope, q, k, pos, q_out, k_out, q_norm=w, k_norm=w)
    alone_q, alone_k = torch.full_like(q_out, 9.0), torch.full_like(k_out, 9.0)
    aoh.aoh_norm_rotate(rope, q, None, pos, alone_q, None, q_norm=w)
    aoh.aoh_norm_rotate(rope, None, k, pos, None, alone_k, k_norm=w)
    assert torch.equal(alone_q, q_out) and torch.equal(alone_k, k_out)
    before = v.clone()
    aoh.aoh_norm_rotate(rope, q, k, pos, q, k, q_norm=w, k_norm=w)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(v, before)
    aoh.aoh_norm_rotate(rope, q[:0], k[:0], pos[:0], q_out[:0], k_out[:0])


def test_bad_numbers_stay_in_their_head():
    n, h, d = 20, 6, 64
    q = randn((n, h, d), 1)
    pos, w = ints(range(n)), weights(d, torch.float32, 0)
    rope = aoh.Rope(32)
    want, spoilt = torch.empty_like(q), torch.empty_like(q)
    aoh.aoh_norm_rotate(rope, q, None, pos, want, None)
    x = q.clone()
    x[3, 2, 5] = float("nan")
    x[7, 1, 50] = float("inf")
    aoh.aoh_norm_rotate(rope, x, None, pos, spoilt, None)
    hit = torch.zeros_like(q, dtype=torch.bool)
    hit[3, 2, 5] = hit[3, 2, 21] = hit[7, 1, 50] = True  # a pair; a number that does not turn
    assert torch.equal(spoilt[~hit], want[~hit])
    assert spoilt[3, 2, [5, 21]].isnan().all() and spoilt[7, 1, 50] == float("inf")
    aoh.aoh_norm_rotate(rope, q, None, pos, want, None, q_norm=w)
    aoh.aoh_norm_rotate(rope, x, None, pos, spoilt, None, q_norm=w)
    rows = torch.zeros(n, h, dtype=torch.bool)
    rows[3, 2] = rows[7, 1] = True
    assert torch.equal(spoilt[~rows], want[~rows])
    assert spoilt[3, 2].isnan().all()


# ------------------------------------------------------------------ into pages

class Pages:
    """A pool with its own view of what lies where."""

    def __init__(self, hq, hkv, d, page, n_pages, form, max_seqs=16):
        self.c = aoh.PagedCache(n_pages, page, hq, hkv, d, 0, 1, [0] * hkv, form=form, max_seqs=max_seqs)
        self.c.pool.fill_(7)
        self.hkv, self.d, self.page, self.n_pages, self.form = hkv, d, page, n_pages, form

    def rows(self, pages, slots):
        """K, V [n, hkv, d] in 64 bits, and their powers [n, 2, hkv] (8 bits)."""
        n = self.n_pages * 2 * self.hkv * self.page * self.d
        shape = (self.n_pages, 2, self.hkv, self.page, self.d)
        if self.form == "bf16":
            x = f64(self.c.pool.view(torch.bfloat16).view(shape))
            return x[pages, 0, :, slots], x[pages, 1, :, slots], None
        codes = self.c.pool[:n].view(shape).cpu().numpy()
        powers = self.c.pool[n:].view(torch.int8).view(self.n_pages, self.hkv, 2, self.page).cpu().numpy()
        e = powers[pages, :, :, slots].transpose(0, 2, 1)
        return tuple(opaged.decode(codes[pages, sel, :, slots], e[:, sel]) for sel in (0, 1)) + (e,)


def check_8bit(got, e, want, size, what):
    _, power = opaged.encode(want)
    most = np.abs(want).max(-1)
    border = np.abs(most / 448.0 / 2.0 ** e.astype(float) - 1) < 2.0 ** -19
    border |= np.abs(most / 448.0 / 2.0 ** power.astype(float) - 1) < 2.0 ** -19
    assert ((e == power) | border).all(), what
    step = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * 2.0 ** e.astype(float)[..., None])
    off = np.abs(got - want) - step - 2.0 ** -20 * size
    assert off.max() <= 0, f"{what}: {off.max():.3e} beyond the tolerance"


PAGED = [
    # rows of each sequence, tokens before, Hq, Hkv, d, page, rotated, interleaved, norms, fused
    ([1], [0], 28, 4, 128, 16, 128, False, None, False),
    ([1, 1, 1], [9, 0, 4096], 8, 2, 64, 64, 64, False, torch.float32, True),
    ([5, 0, 130, 17], [3, 50, 0, 4000], 32, 8, 128, 64, 128, False, torch.bfloat16, True),
    ([300, 2], [15, 16], 16, 1, 128, 128, 64, True, None, False),
    ([40, 1, 700], [0, 1, 33], 6, 3, 64, 32, 32, False, torch.float32, False),
    ([2900, 10], [100, 7], 8, 8, 128, 16, 128, False, torch.bfloat16, True),
    ([1500], [0], 24, 12, 64, 16, 64, True, None, True),
]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(PAGED)))
def test_into_pages(case, form):
    rows, before, hq, hkv, d, page, rotated, il, wt, fused = PAGED[case]
    n, after = sum(rows), [a + b for a, b in zip(rows, before)]
    q, k, v = inputs(n, hq, hkv, d, fused, 31 * case)
    width = max(-(-m // page) for m in after)
    n_pages = width * len(rows) + 3
    order = np.random.default_rng(case).permutation(n_pages)[:width * len(rows)].reshape(len(rows), width)
    p = Pages(hq, hkv, d, page, n_pages, form)
    pool_before = p.c.pool.clone()
    freqs = orot.frequencies(rotated, 1e4)
    rope = aoh.Rope(inv_freq=freqs, interleaved=il, scale=1.5)
    wq, wk = weights(d, wt, 1), weights(d, wt, 2)
    q_out = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda")
    cu = None if all(r == 1 for r in rows) else ints(np.concatenate([[0], np.cumsum(rows)]))
    p.c.append_rotated(rope, q, k, v, ints(after), ints(order), q_out, cu_rows=cu, q_norm=wq, k_norm=wk, eps=1e-4)
    p.c.check()
    pos = np.concatenate([np.arange(b, b + r) for b, r in zip(before, rows)])
    seq = np.repeat(np.arange(len(rows)), rows)
    want, size = definition(q, wq, 1e-4, pos, freqs, il, 1.5)
    close(q_out, want, size, f"q of case {case}")
    kk, vv, e = p.rows(order[seq, pos // page], pos % page)
    want, size = definition(k, wk, 1e-4, pos, freqs, il, 1.5)
    if form == "bf16":
        close(torch.from_numpy(kk), want, size, f"k of case {case}")
        assert np.array_equal(vv, f64(v))
    else:
        check_8bit(kk, e[:, 0], want, size, f"k of case {case}")
        codes, power = opaged.encode(f64(v))
        assert np.array_equal(vv, opaged.decode(codes, power)) and np.array_equal(e[:, 1], power)
    # what no row was written to is as it was: the same rows appended to a copy, then wiped there
    wiped = p.c.pool.clone()
    for x in (wiped, pool_before):
        bytes_ = 2 if form == "bf16" else 1
        m = n_pages * 2 * hkv * page * d * bytes_
        view = x[:m].view(n_pages, 2, hkv, page, d * bytes_)
        view[order[seq, pos // page], :, :, pos % page] = 0
        if form == "e4m3":
            x[m:].view(n_pages, hkv, 2, page)[order[seq, pos // page], :, :, pos % page] = 0
    assert torch.equal(wiped, pool_before)


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_same_as_rotating_first(form):
    """v and, in bf16, k land as an append of rotated rows puts them; positions of the caller's
    are those that count."""
    rows, hq, hkv, d, page = [30, 9], 8, 2, 128, 32
    q, k, v = inputs(39, hq, hkv, d, True, 5)
    pos = ints(far_positions(39, 4))
    rope = aoh.Rope(d)
    table, lens, cu = ints([[3, 1], [0, 2]]), ints([35, 9]), ints([0, 30, 39])
    a, b = (Pages(hq, hkv, d, page, 5, form) for _ in range(2))
    q1, q2, k2 = torch.empty((39, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((39, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((39, hkv, d), dtype=torch.bfloat16, device="cuda")
    a.c.append_rotated(rope, q, k, v, lens, table, q1, cu_rows=cu, positions=pos)
    aoh.aoh_norm_rotate(rope, q, k, pos, q2, k2)
    b.c.append(k2, v, lens, table, cu_rows=cu)
    for c in (a.c, b.c):
        c.check()
    assert torch.equal(q1, q2)
    if form == "bf16":
        assert torch.equal(a.c.pool, b.c.pool)
    # and q in place
    a.c.append_rotated(rope, q, k, v, lens, table, q, cu_rows=cu, positions=pos)
    assert torch.equal(q, q1)


def test_rows_without_a_place_are_left_alone():
    hq, hkv, d, page = 4, 2, 64, 16
    for form in ("bf16", "e4m3"):
        p = Pages(hq, hkv, d, page, 4, form)
        before = p.c.pool.clone()
        rope = aoh.Rope(d)
        q, k, v = inputs(3, hq, hkv, d, False, 6)
        # a slot without a request: nothing, and no error
        q_out = torch.full((3, hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
        p.c.append_rotated(rope, q, k, v, ints([0, 0, 0]), ints([[0], [1], [2]]), q_out)
        p.c.check()
        assert torch.equal(p.c.pool, before) and (q_out == 5).all()
        # past the table; rows that cu_rows gives to no sequence; more rows than tokens
        for lens, cu in (([17, 0, 0], None), ([1, 1, 0], [0, 1, 2, 2]), ([0, 1, 1], [0, 1, 2, 3])):
            q_out.fill_(5)  # (the call before has written the other rows)
            p.c.append_rotated(rope, q, k, v, ints(lens), ints([[3], [1], [2]]), q_out, cu_rows=None if cu is None else ints(cu))
            with pytest.raises(aoh.AohError, match="out of range"):
                p.c.check()
            lost = 0 if lens[0] in (17, 0) else 2
            assert (q_out[lost] == 5).all()
        # a page out of range: q alone
        p.c.pool.copy_(before)
        p.c.append_rotated(rope, q, k, v, ints([1, 1, 1]), ints([[4], [-1], [1 << 30]]), q_out)
        with pytest.raises(aoh.AohError, match="out of range"):
            p.c.check()
        assert torch.equal(p.c.pool, before) and not (q_out == 5).all(-1).all(-1).any()


def test_rows_that_are_not_finite_in_8_bits():
    """An infinity or NaN becomes the NaN code, beside finite numbers as they are; largest numbers stay
    finite; a row of zeros has the least power."""
    hq, hkv, d, page = 1, 1, 64, 16
    k = torch.ones((5, 1, d), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 40] = float("inf")
    k[1, 0, 40] = float("nan")
    k[2] = 0
    k[3] *= 3.0e38
    k[4, 0, 40] = -float("inf")
    p = Pages(hq, hkv, d, page, 1, "e4m3")
    q = torch.zeros_like(k)
    p.c.append_rotated(aoh.Rope(0), q, k, k, ints([5]), ints([[0]]), torch.empty_like(q), cu_rows=ints([0, 5]))
    p.c.check()
    kk, vv, e = p.rows(np.zeros(5, int), np.arange(5))
    codes, power = opaged.encode(f64(k))
    want = opaged.decode(codes, power)
    assert np.array_equal(kk, want, equal_nan=True) and np.array_equal(vv, want, equal_nan=True)
    assert np.array_equal(e, np.stack([power, power], 1))


def test_captured_and_on_another_stream():
    """A graph reads lengths, table and positions when it is replayed."""
    hq, hkv, d, page = 8, 2, 128, 16
    p = Pages(hq, hkv, d, page, 8, "e4m3")
    rope, w = aoh.Rope(d), weights(d, torch.bfloat16, 0)
    q, k, v = inputs(2, hq, hkv, d, False, 8)
    lens, table, q_out = ints([1, 1]), ints([[0, 1], [2, 3]]), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        p.c.append_rotated(rope, q, k, v, lens, table, q_out, q_norm=w, k_norm=w)
    for n in ([5, 1], [31, 32]):
        lens.copy_(ints(n))
        q.copy_(randn(tuple(q.shape), sum(n)))
        graph.replay()
        want, size = definition(q, w, 1e-6, [x - 1 for x in n], orot.frequencies(d, 1e4), False, 1.0)
        close(q_out, want, size, f"lengths {n}")
    p.c.check()
    side = torch.empty_like(q)
    s.wait_stream(torch.cuda.current_stream())
    aoh.aoh_norm_rotate(rope, q, k, ints([30, 31]), side, torch.empty_like(k), q_norm=w, k_norm=w, stream=s)
    s.synchronize()
    assert torch.equal(side, q_out)
