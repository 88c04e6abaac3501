"""Attention of chunks over pages against its 64-bit definition (oracle.paged) on what the
pages hold.

Tolerance: as for packed prompts (test_gpu_paged.py): rounding each softmax weight to 8 significant
bits moves an output by at most 2^-9 * sum_j p_j |v_j| (``mag``, the definition run on |v|), storing it
as bf16 by 2^-9 |o|; twice both plus 1e-4 is allowed (gpu_cases.assert_matches). Rows of 8 bits
reach the tensor cores as the bf16 numbers that they stand for, so nothing else is added."""

import numpy as np
import pytest
import torch

from gpu_cases import assert_matches, ensure_lib, f64
from oracle import paged as opaged
from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


def randn(shape, seed, spread=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    return (x * torch.exp2(spread * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))).bfloat16()


def ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def sums(xs):
    return np.concatenate([[0], np.cumsum(xs)]).tolist()


def held(x, form):
    return f64(x) if form == "bf16" else opaged.decode(*opaged.encode(f64(x)))


class Case:
    """Sequences of k_lens tokens in pages of a random order, and queries for their last q_lens."""

    def __init__(self, q_lens, k_lens, hq, hkv, d, labels, sink, window, page, form, seed=0, fused=False, spread=0.0):
        self.q_lens, self.k_lens, self.labels, self.sink, self.window, self.form = q_lens, k_lens, labels, sink, window, form
        n, m = sum(q_lens), sum(k_lens)
        self.q = randn((n, hq, d), seed)
        if fused:
            self.q = torch.cat([self.q, randn((n, 2 * hkv, d), seed + 5)], 1)[:, :hq]
        self.k, self.v = randn((m, hkv, d), seed + 1, spread), randn((m, hkv, d), seed + 2, spread)
        width = max(1, max(-(-x // page) for x in k_lens))
        need = sum(-(-x // page) for x in k_lens)
        order = np.random.default_rng(seed).permutation(need + 3)
        table = np.full((len(k_lens), width), -7, dtype=np.int32)
        at = 0
        for b, x in enumerate(k_lens):
            c = -(-x // page)
            table[b, :c] = order[at:at + c]
            at += c
        self.c = aoh.PagedCache(need + 3, page, hq, hkv, d, sink, window, labels, form=form, max_seqs=len(q_lens))
        self.c.pool.fill_(255)  # NaN wherever nothing is written
        self.table, self.lens = ints(table), ints(k_lens)
        if m:
            self.c.append(self.k, self.v, self.lens, self.table, cu_rows=ints(sums(k_lens)))
        self.c.check()
        self.out = torch.full((n, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.formed = {}

    def attend(self, **kw):
        self.c.attend(self.q, self.q_lens, self.lens, self.table, self.out, **kw)
        self.c.check()
        return self.out

    def held(self, b, keys):
        """What the pages hold of sequence b, formed once for the same k and v."""
        version = (self.k._version, self.v._version)
        if self.form == "bf16" or self.formed.get("version") != version:
            self.formed = {"version": version}
        if b not in self.formed:
            self.formed[b] = held(self.k[keys], self.form), held(self.v[keys], self.form)
        return self.formed[b]

    def matches(self, what, sequences=None):
        qs, ks = sums(self.q_lens), sums(self.k_lens)
        q, out = f64(self.q), f64(self.out)
        for b in range(len(self.q_lens)) if sequences is None else sequences:
            if self.q_lens[b] == 0:
                continue
            rows, keys = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            k, v = self.held(b, keys)
            want = opaged.attend(q[rows], k, v, self.labels, self.sink, self.window)
            mag = opaged.attend(q[rows], k, np.abs(v), self.labels, self.sink, self.window)
            assert_matches(out[rows], want, f"{what}, sequence {b}", mag=mag, abs_bounds=False)


CASES = [
    # q_lens, k_lens, Hq, Hkv, d, labels, sink, window, page
    ([1], [1], 2, 1, 64, [0], 0, 1, 16),
    ([5], [5], 4, 4, 128, [0, 1, 0, 1], 0, 1, 64),
    ([1, 128, 0, 129, 127, 300], [1, 128, 7, 129, 127, 300], 8, 2, 128, [0, 1], 4, 40, 32),
    ([77, 1, 513, 64], [77, 900, 600, 64], 8, 2, 64, [1, 0], 0, 130, 16),
    ([600, 257], [700, 258], 7, 1, 128, [1], 200, 30, 128),
    ([1300], [1300], 14, 2, 128, [0, 1], 128, 256, 64),
    ([90, 1, 200], [400, 1000, 200], 6, 2, 128, [0, 1], 16, 100, 16),
    ([33, 5], [1290, 129], 16, 1, 64, [0], 0, 1, 32),
    # fewer positions than rows, and none
    ([300, 7, 130], [10, 0, 131], 4, 2, 128, [0, 1], 2, 3, 16),
    ([9, 260], [0, 0], 4, 2, 64, [0, 1], 2, 3, 64),
    # many sequences (lengths that travel by way of the device), and few rows of each
    ([3 + 5 * (i % 7) for i in range(70)], [60 + 5 * (i % 7) for i in range(70)], 4, 2, 64, [0, 1], 8, 9, 16),
    ([1 + i % 5 for i in range(90)], [1 + i % 5 + 37 * i for i in range(90)], 32, 8, 128, [0, 1] * 4, 20, 300, 64),
    ([140 + 31 * (i % 5) for i in range(20)], [140 + 31 * (i % 5) + i for i in range(20)], 24, 8, 128, [0, 1] * 4, 8, 100, 32),
    # few rows after long prefixes: shared by clusters
    ([17, 3, 1], [3000, 2999, 1], 32, 8, 64, [0, 1] * 4, 10, 500, 64),
    ([33, 20], [2500, 900], 7, 1, 128, [0], 0, 1, 16),
    ([5, 100, 26], [2049, 10, 1500], 10, 2, 128, [0, 1], 100, 300, 128),
    ([16, 9], [1900, 1281], 16, 1, 128, [0], 0, 1, 32),
    ([1, 1, 1, 1], [5000, 100, 1, 640], 8, 1, 128, [0], 0, 1, 16),
    ([3, 1], [9000, 257], 4, 1, 128, [0], 0, 1, 64),
    ([100], [7003], 4, 2, 128, [0, 0], 0, 1, 16),
    ([2, 11], [6300, 1], 16, 2, 64, [0, 1], 300, 3000, 16),
    ([5], [4000], 2, 2, 64, [0, 1], 7, 90, 128),
    ([300, 40], [3333, 2600], 3, 3, 128, [0, 1, 0], 0, 1000, 64),
    ([311], [2900], 16, 4, 128, [0, 0, 1, 0], 5, 900, 32),
    # a window that begins inside of the sinks' last tile, and behind a gap
    ([70], [1111], 6, 2, 128, [1, 1], 128, 129, 16),
    ([4], [2000], 40, 8, 64, [1] * 8, 130, 63, 16),
    # several waves of items
    ([1400, 900], [1700, 901], 16, 8, 64, [0, 1] * 4, 3, 700, 64),
    ([2100], [2500], 32, 8, 128, [0, 1] * 4, 64, 600, 64),
]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_chunks(case, form):
    c = Case(*CASES[case], form, seed=10 * case, fused=case % 2 == 1, spread=1.5 if case % 3 == 0 else 0.0)
    # the host's idea of the lengths: right, none, too short, too long
    hint = [c.k_lens, None, [x // 3 for x in c.k_lens], [x + 4000 for x in c.k_lens]][case % 4]
    c.attend(k_lens=hint)
    c.matches(f"chunks {case}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_many_items_in_several_launches(form):
    c = Case([40] * 110, [50] * 110, 64, 64, 64, [0] * 64, 0, 1, 16, form)
    c.attend()
    c.matches("many items", [0, 48, 49, 50, 51, 99, 100, 101, 109])
    assert torch.isfinite(c.out.float()).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_as_a_single_token(form, d):
    """One row a sequence is what the decode gives."""
    lens = [1, 700, 33, 2048, 129]
    c = Case([1] * 5, lens, 8, 2, d, [0, 1], 10, 100, 16, form, seed=3)
    c.attend(k_lens=lens)
    c.matches("single tokens")
    other = torch.empty_like(c.out)
    c.c.decode(c.q, c.lens, c.table, other)
    c.c.check()
    assert (f64(other) - f64(c.out)).max() < 0.02


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_neighbours_and_free_pages_are_not_seen(form):
    """NaN in other sequences' pages, in free ones and behind a sequence's end changes nothing."""
    c = Case([70, 200, 33], [75, 300, 633], 8, 2, 128, [0, 1], 4, 50, 64, form, seed=5)
    first = c.attend(k_lens=c.k_lens).clone()
    k = torch.full((300, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.c.append(k, k, ints([0, 300, 0]), c.table, cu_rows=ints([0, 0, 300, 300]))
    c.out.fill_(float("nan"))
    c.attend(k_lens=c.k_lens)
    assert torch.equal(c.out[:70], first[:70]) and torch.equal(c.out[270:], first[270:])


SPOILT = [CASES[i] for i in (2, 3, 5, 6, 13, 14, 17, 20, 22, 24)]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(SPOILT)))
def test_spoilt_keys_reach_the_rows_that_see_them(case, form):
    """K and V of some positions NaN (or infinite, which 8 bits hold as NaN): the rows that see them
    are NaN, the others as they would be without."""
    c = Case(*SPOILT[case], form, seed=7 * case)
    clean = c.attend(k_lens=c.k_lens).clone()
    g = np.random.default_rng(case)
    ks, bad = sums(c.k_lens), []
    k, v = c.k.clone(), c.v.clone()
    for b, m in enumerate(c.k_lens):
        at = sorted(set(g.integers(max(0, m - c.q_lens[b] - 20), m, 2))) if m else []
        bad.append(at)
        for j in at:
            k[ks[b] + j] = float("nan")
            v[ks[b] + j] = float("inf") if case % 2 else float("nan")
    c.c.append(k, v, c.lens, c.table, cu_rows=ints(ks))
    c.out.fill_(0)
    out = f64(c.attend(k_lens=c.k_lens))
    qs, clean = sums(c.q_lens), f64(clean)
    hq, hkv = c.q.shape[1], len(c.labels)
    for b, (n, m) in enumerate(zip(c.q_lens, c.k_lens)):
        pos = np.arange(m - n, m)[:, None]
        j = np.array(bad[b], dtype=int)[None, :]
        for h in range(hq):
            see = j <= pos
            if c.labels[h // (hq // hkv)]:
                see &= (j < c.sink) | (pos - j < c.window)
            hit = see.any(1)
            rows = np.arange(qs[b], qs[b + 1])
            assert np.isnan(out[rows[hit], h]).all(), (b, h)
            # (rows that are gone over again are summed in another order)
            d = np.abs(out[rows[~hit], h] - clean[rows[~hit], h])
            assert (d <= 2.0 ** -6 * np.abs(clean[rows[~hit], h]) + 0.02).all(), (b, h, d.max())


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_out_of_range(form):
    """Pages and lengths out of range are reported; other sequences are right all the same."""
    c = Case([20, 30], [150, 600], 8, 2, 128, [0, 1], 4, 50, 32, form, seed=2)
    good = c.table.clone()
    for page in (-1, c.c.n_pages, 2 ** 31 - 1):
        c.table.copy_(good)
        c.table[0, 3] = page
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
        with pytest.raises(aoh.AohError, match="out of range"):
            c.c.check()
        c.matches(f"page {page}", [1])
    c.table.copy_(good)
    for n in (-5, good.shape[1] * 32 + 1, 2 ** 31 - 1):
        c.lens.copy_(ints([n, 600]))
        c.table[0, :] = 0  # (of a length past the table all of it is read)
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
        with pytest.raises(aoh.AohError, match="out of range"):
            c.c.check()
        c.matches(f"length {n}", [1])
        if n < 0:
            assert (c.out[:20] == 0).all()


def test_large_and_tiny_rows():
    """8-bit rows of any size: the scores of K rows of 2^-60 to 2^6, V rows of 2^-70 to 2^90."""
    for d in (64, 128):
        c = Case([1, 40], [300, 700], 4, 2, d, [0, 1], 3, 90, 16, "e4m3", seed=d)
        e = torch.linspace(-70, 90, c.v.shape[0], device="cuda")[torch.randperm(c.v.shape[0], device="cuda")]
        c.v = (c.v.float() * torch.exp2(e.round()).view(-1, 1, 1)).bfloat16()
        e = torch.linspace(-60, 6, c.k.shape[0], device="cuda")
        c.k = (c.k.float() * torch.exp2(e.round()).view(-1, 1, 1)).bfloat16()
        c.c.append(c.k, c.v, c.lens, c.table, cu_rows=ints(sums(c.k_lens)))
        c.attend(k_lens=c.k_lens)
        c.matches(f"d {d}")


def test_captured_over_growing_lengths():
    """A graph of append and attend reads lengths and table at replay: two calls of one handle, three
    drafted tokens a step, a slot whose request ends."""
    hq, hkv, d, page, form = 8, 2, 128, 16, "e4m3"
    rope = aoh.Rope(d)
    c = aoh.PagedCache(40, page, hq, hkv, d, 4, 40, [0, 1], form=form, max_seqs=2)
    table, lens, cu = ints(np.arange(40).reshape(2, 20)), ints([0, 0]), ints([0, 3, 6])
    q, k, v = randn((6, hq, d), 0), randn((6, hkv, d), 1), randn((6, hkv, d), 2)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(3)
        c.append_rotated(rope, q, k, v, lens, table, turned, cu_rows=cu)
        c.attend(turned, [3, 3], lens, table, out)
    freqs = orot.frequencies(d, 1e4)
    past = [[np.zeros((0, hkv, d))] * 2 for _ in range(2)]
    for step in range(30):
        for i, x in enumerate((q, k, v)):
            x.copy_(randn(tuple(x.shape), 100 * step + i))
        graph.replay()
        assert lens.tolist() == [3 * step + 3] * 2
        for b in range(2):
            rows, pos = slice(3 * b, 3 * b + 3), np.arange(3 * step, 3 * step + 3)
            kk = opaged.decode(*opaged.encode(orot.rotate(f64(k[rows]), pos, freqs)))
            past[b] = [np.concatenate([past[b][0], kk]), np.concatenate([past[b][1], held(v[rows], form)])]
            if step % 7 == 6:
                want = opaged.attend(f64(turned[rows]), past[b][0], past[b][1], [0, 1], 4, 40)
                mag = opaged.attend(f64(turned[rows]), past[b][0], np.abs(past[b][1]), [0, 1], 4, 40)
                # a K number whose 32-bit rotation falls on the other side of a border of its codes is a step
                # off, 2^-4 of its row's largest at most: rarely, and in one number of a row
                assert_matches(f64(out[rows]), want, f"step {step}", mag=mag, abs_bounds=False)
    c.check()
    lens.fill_(-3)  # the next step's lengths are 0: slots without a request
    c.attend(turned, [3, 3], ints([0, 0]), table, out)
    c.check()
    assert (out == 0).all()


def test_on_another_stream():
    c = Case([40, 3], [400, 1000], 8, 2, 64, [0, 1], 4, 50, 64, "bf16", seed=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, stream=s)
    s.synchronize()
    c.matches("another stream")


def test_same_results_again():
    c = Case([40, 3, 300], [4000, 9000, 2500], 8, 2, 128, [0, 1], 4, 2000, 64, "e4m3", seed=1)
    first = c.attend(k_lens=c.k_lens).clone()
    for _ in range(5):
        c.out.fill_(float("nan"))
        assert torch.equal(c.attend(k_lens=c.k_lens), first)


WRITTEN_OUT = [
    # calls whose items visit the same tiles often: 8-bit pages are written out as bf16 ones first
    ([1500], [4100], 16, 4, 128, [0, 1, 0, 0], 20, 700, 16),
    ([900, 1, 2000], [900, 700, 2100], 16, 2, 64, [0, 1], 130, 500, 64),
    ([700, 650, 800], [5000, 660, 2500], 32, 8, 128, [0, 1] * 4, 64, 512, 128),
]


@pytest.mark.parametrize("case", range(len(WRITTEN_OUT)))
def test_pages_written_out_first(case):
    """Right for whatever lengths the host takes the sequences to have, and so are those of the kernel that
    decodes them itself (a captured call takes no memory, so it is that one)."""
    c = Case(*WRITTEN_OUT[case], "e4m3", seed=50 + case, fused=True, spread=1.0)
    c.attend(k_lens=c.k_lens)
    c.matches("written out")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
    c.out.fill_(float("nan"))
    graph.replay()
    c.c.check()
    c.matches("captured")
    for hint in ([n // 2 for n in c.k_lens], [c.k_lens[0] // 3] + c.k_lens[1:], [n + 1000 for n in c.k_lens], None,
                 [0] + c.k_lens[1:]):
        c.out.fill_(float("nan"))
        c.attend(k_lens=hint)
        c.matches(f"hint {hint}")


def test_bad_pages_written_out_first():
    c = Case([900, 800], [2000, 3000], 16, 4, 128, [0, 1, 0, 0], 20, 700, 32, "e4m3", seed=2)
    first = c.attend(k_lens=c.k_lens).clone()
    good = c.table.clone()
    for page in (-1, c.c.n_pages):
        c.table.copy_(good)
        c.table[0, 3] = page
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
        with pytest.raises(aoh.AohError, match="out of range"):
            c.c.check()
        assert torch.equal(c.out[900:], first[900:])
    # NaN where nothing is visible: behind a sequence's end, and between sinks and windows
    c.table.copy_(good)
    k, v = c.k.clone(), c.v.clone()
    k[1000], v[1000] = float("nan"), float("nan")  # position 1000 of the first: before its rows, 1100 .. 1999
    c.c.append(k, v, c.lens, c.table, cu_rows=ints(sums(c.k_lens)))
    out = c.attend(k_lens=c.k_lens)
    hidden = torch.zeros((900, 16), dtype=torch.bool, device="cuda")
    hidden[600:, 4:8] = True  # KV head 1 streams: rows from position 1100 + 600 = 1700 on see 1001 on
    assert out[:900][~hidden].isnan().all() and not out[:900][hidden].isnan().any()
    assert torch.equal(out[900:], first[900:])


def test_written_out_pages_are_what_the_codes_stand_for():
    """Of whole items in both, so that the outputs are equal bit by bit."""
    c = Case([300] * 20, [450 + i for i in range(20)], 16, 4, 128, [0, 1, 0, 0], 20, 200, 16, "e4m3", seed=57, spread=1.0)
    first = c.attend(k_lens=c.k_lens).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
    c.out.fill_(float("nan"))
    graph.replay()
    c.c.check()
    assert torch.equal(c.out, first)


@pytest.mark.parametrize("n", [63, 64, 100])
def test_pages_of_many_sequences_written_out(n):
    """Lists of sequences that travel by value or by way of the device, some without rows or keys and some
    longer than the host takes them to be."""
    q_lens = [0 if i % 13 == 5 else 290 + 7 * (i % 6) for i in range(n)]
    k_lens = [0 if i % 17 == 3 else q + 61 * (i % 9) for i, q in enumerate(q_lens)]
    hint = [max(0, k - 200) if i % 11 == 2 else k for i, k in enumerate(k_lens)]
    c = Case(q_lens, k_lens, 16, 2, 128, [0, 1], 10, 260, 32, "e4m3", seed=70 + n)
    c.attend(k_lens=hint)
    c.matches(f"{n} sequences written out")


def test_written_out_after_an_append_in_flight():
    """An append and the attention that follow each other without a wait: the new rows are seen."""
    c = Case([1200], [3000], 16, 4, 128, [0, 1, 0, 0], 20, 700, 32, "e4m3", seed=9)
    for step in range(6):
        c.k.copy_(randn(tuple(c.k.shape), 100 + step))
        c.v.copy_(randn(tuple(c.v.shape), 200 + step))
        torch.cuda.synchronize()
        c.c.append(c.k, c.v, c.lens, c.table, cu_rows=ints(sums(c.k_lens)))
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
        if step % 3 == 2:
            c.matches(f"step {step}")
    c.c.check()


FEW = [
    # a few rows a sequence: parts of it beside one another on the decode kernel
    # q_lens, k_lens, Hq, Hkv, d, labels, sink, window, page
    ([4, 1, 3, 2], [4, 500, 2000, 131], 8, 2, 128, [0, 1], 3, 40, 16),
    ([5], [3000], 28, 4, 128, [1, 0, 0, 1], 16, 300, 64),
    ([3, 5, 2], [900, 5, 40], 16, 1, 64, [0], 0, 1, 32),
    ([8, 7], [1030, 260], 4, 2, 64, [1, 0], 100, 129, 128),
    ([16, 11], [400, 6000], 3, 3, 128, [0, 1, 1], 5, 64, 16),
    # fewer positions than rows, and none
    ([4, 3, 2, 4], [2, 0, 1, 0], 8, 2, 64, [0, 1], 3, 40, 16),
    # more parts than travel by value, windows that move within a part
    ([1 + i % 4 for i in range(80)], [1 + i % 4 + 53 * (i % 11) for i in range(80)], 32, 8, 128, [0, 1] * 4, 2, 3, 16),
    ([6] * 30, [40 + 97 * (i % 13) for i in range(30)], 24, 8, 64, [1, 0] * 4, 0, 5, 64),
    ([2] * 20, [9000 + i for i in range(20)], 32, 8, 64, [0] * 8, 0, 1, 64),
    ([6] * 3, [40, 1007, 300], 24, 8, 64, [1, 0] * 4, 0, 5, 64),
    ([1 + i % 4 for i in range(80)], [2400 + 3 * i for i in range(80)], 8, 2, 128, [0, 0], 0, 1, 64),
]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(FEW)))
def test_few_rows(case, form):
    c = Case(*FEW[case], form, seed=300 + case, fused=case % 2 == 0, spread=1.5)
    # (calls of one part a sequence run there by the last, others of a few parts by the one before)
    for hint in (c.k_lens, [0] * len(c.k_lens), [1 << 17] * len(c.k_lens)):
        c.out.fill_(float("nan"))
        c.attend(k_lens=hint)
        c.matches(f"few rows {case}, hint {hint[:3]}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(FEW)))
def test_spoilt_keys_among_few_rows(case, form):
    """K and V that are not finite at the rows' own positions and around the beginnings of their windows reach
    the rows that see them, and no other of the same sequence."""
    c = Case(*FEW[case], form, seed=400 + case)
    hint = [1 << 17 if max(c.q_lens) * (c.q.shape[1] // len(c.labels)) <= 16 else 0] * len(c.k_lens)
    clean = f64(c.attend(k_lens=hint))
    ks, qs, hkv = sums(c.k_lens), sums(c.q_lens), len(c.labels)
    G = c.q.shape[1] // hkv
    for what in ("v nan", "v inf", "k nan"):
        k, v, bad = c.k.clone(), c.v.clone(), []
        for b, (n, m) in enumerate(zip(c.q_lens, c.k_lens)):
            # the last rows' keys but the very last; a key that leaves the window within the chunk
            at = sorted({p for p in (m - 1 - n // 2, m - n - c.window + 2, m - 2) if 0 <= p < m - 1})[:1 + (case + b) % 3]
            bad.append(at)
            for j in at:
                (k if what == "k nan" else v)[ks[b] + j, :, (j * 7) % c.q.shape[2]] = float("inf" if what == "v inf" else "nan")
        c.c.append(k, v, c.lens, c.table, cu_rows=ints(ks))
        c.out.fill_(0)
        out = f64(c.attend(k_lens=hint))
        for b, (n, m) in enumerate(zip(c.q_lens, c.k_lens)):
            pos, j = np.arange(m - n, m)[:, None], np.array(bad[b], dtype=int)[None, :]
            for h in range(c.q.shape[1]):
                see = j <= pos
                if c.labels[h // G]:
                    see &= (j < c.sink) | (pos - j < c.window)
                rows, hit = np.arange(qs[b], qs[b + 1]), see.any(1)
                got = out[rows, h]
                if what == "k nan":
                    assert np.isnan(got[hit]).all(), (what, b, h)
                elif hit.any():
                    assert not np.isfinite(got[hit]).all(1).any(), (what, b, h)
                ok = clean[rows[~hit], h]
                # (rows that are gone over again are summed in another order; 8-bit codes of a row whose largest
                # number became an infinity are those of its other numbers)
                if form == "bf16" or what != "v inf":
                    assert (np.abs(got[~hit] - ok) <= 2.0 ** -6 * np.abs(ok) + 0.02).all(), (what, b, h)
                else:
                    assert np.isfinite(got[~hit]).all(), (what, b, h)
        c.c.append(c.k, c.v, c.lens, c.table, cu_rows=ints(ks))


def test_two_handles_on_two_streams():
    """Written-out pages of two handles' calls that run at once lie apart."""
    cases = [Case([900], [2500], 16, 4, 128, [0, 1, 0, 0], 20, 700, 32, "e4m3", seed=s) for s in (61, 62)]
    wants = [c.attend(k_lens=c.k_lens).clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = [[torch.full_like(c.out, float("nan")) for _ in range(8)] for c in cases]
    torch.cuda.synchronize()
    for i in range(8):
        for c, s, o in zip(cases, streams, outs):
            c.c.attend(c.q, c.q_lens, c.lens, c.table, o[i], k_lens=c.k_lens, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(wants, outs):
        assert all(torch.equal(w, x) for x in o)


MANY = [
    # many short items, which one pipeline an SM goes through: q_lens, k_lens, Hq, Hkv, d, labels, sink, window, page
    ([1 + 7 * i % 60 for i in range(64)], [1 + 7 * i % 60 + 37 * (i % 9) for i in range(64)], 32, 8, 64, [0, 1] * 4, 4, 50, 16),
    # without rows, without keys, fewer positions than rows
    ([(i % 7) * 6 for i in range(90)], [0 if i % 5 == 1 else 13 * (i % 23) for i in range(90)], 32, 8, 128, [1, 0] * 4, 9, 70, 32),
    ([1 + 11 * (i % 29) for i in range(60)], [1 + 11 * (i % 29) + 61 * (i % 4) for i in range(60)], 8, 8, 128, [0] * 7 + [1], 0, 130, 128),
    ([40 + i % 3 for i in range(70)], [40 + i % 3 + 128 * (i % 5) for i in range(70)], 24, 8, 64, [0, 0, 1, 1] * 2, 130, 200, 64),
]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_short_items(case, form):
    c = Case(*MANY[case], form, seed=500 + case, fused=case % 2 == 0, spread=1.0)
    for hint in (c.k_lens, [0] * len(c.k_lens), [n // 2 for n in c.k_lens]):
        c.out.fill_(float("nan"))
        c.attend(k_lens=hint)
        c.matches(f"many short items {case}, hint {hint[:3]}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_bad_sequences_among_many_short_items(d, form):
    """V rows that are NaN reach the rows that see them and no others; lengths and pages out of range are told, and the
    other sequences' rows are what they were."""
    n, past = 70, 150
    q_lens, labels, sink, window = [33] * n, [0, 1] * 4, 5, 60
    c = Case(q_lens, [past + 33] * n, 32, 8, d, labels, sink, window, 16, form, seed=8 + d)
    clean = c.attend(k_lens=c.k_lens).clone()
    v = c.v.clone().view(n, past + 33, 8, d)
    at = {3: past + 20, 41: past - 10, 69: 2}  # sequence: position
    for b, p in at.items():
        v[b, p] = float("nan")
    c.c.append(c.k, v.view(-1, 8, d), c.lens, c.table, cu_rows=ints(sums(c.k_lens)))
    got = c.attend(k_lens=c.k_lens).view(n, 33, 8, 4, d)
    want = clean.view(n, 33, 8, 4, d)
    pos = torch.arange(past, past + 33, device="cuda")
    for b in range(n):
        for h in range(8):
            sees = torch.zeros(33, dtype=torch.bool, device="cuda")
            if b in at:
                sees = at[b] <= pos
                if labels[h] and at[b] >= sink:
                    sees = sees & (pos - at[b] < window)
            assert got[b, sees, h].isnan().all(), (b, h)
            x, y = got[b, ~sees, h].double(), want[b, ~sees, h].double()
            # rows that are gone over again are summed in another order: two roundings to bf16, of weights and of sums
            assert ((x - y).abs() <= 2.0 ** -6 * y.abs() + 0.02).all(), (b, h)
    c.c.append(c.k, c.v, c.lens, c.table, cu_rows=ints(sums(c.k_lens)))
    table, lens = c.table.clone(), c.lens.clone()
    for what in ("page", "long", "negative"):
        c.table.copy_(table)
        c.lens.copy_(lens)
        if what == "page":
            c.table[17, 4] = c.c.n_pages
        else:
            c.lens[17] = 1 << 20 if what == "long" else -5
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
        with pytest.raises(aoh.AohError, match="out of range"):
            c.c.check()
        keep = torch.arange(n * 33, device="cuda") // 33 != 17
        assert torch.equal(c.out[keep], clean[keep]), what


JOINED = [
    # chunks after long prefixes whose items are cut into parts of CTAs of their own, or shared by clusters: q_lens, k_lens, Hq, Hkv, d,
    # labels, sink, window, page
    ([300], [20300], 32, 8, 64, [0, 1] * 4, 64, 512, 64),
    ([600], [6600], 32, 8, 128, [0, 1] * 4, 64, 512, 128),
    ([700], [4700], 12, 3, 128, [0, 1, 0], 20, 500, 16),
    ([700], [20700], 12, 3, 128, [0, 1, 0], 20, 500, 16),
]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(JOINED)))
def test_items_in_parts(case, form):
    """Right for whatever lengths the host takes the sequences to have (parts without a tile, others that the plan
    does not cut), the same numbers every time, and no rows but those that see a spoilt key are spoilt."""
    c = Case(*JOINED[case], form, seed=600 + case, fused=case % 2 == 0, spread=0.5)
    first = c.attend(k_lens=c.k_lens).clone()
    c.matches(f"items in parts {case}")
    for _ in range(3):
        c.out.fill_(float("nan"))
        assert torch.equal(c.attend(k_lens=c.k_lens), first)
    for n in (c.k_lens[0] // 3, c.k_lens[0] + 900):
        c.out.fill_(float("nan"))
        c.attend(k_lens=[n])
        c.matches(f"items in parts {case}, hint {n}")
    # fewer tokens than the host takes it to have: parts without a tile
    c.lens.copy_(ints([c.q_lens[0] + 140]))
    short = c.attend(k_lens=c.k_lens).clone()
    c.lens.copy_(ints(c.k_lens))
    d = Case([c.q_lens[0]], [c.q_lens[0] + 140], *JOINED[case][2:], form, seed=1)
    d.q = c.q
    d.c.append(c.k[:d.k_lens[0]], c.v[:d.k_lens[0]], d.lens, d.table, cu_rows=ints([0, d.k_lens[0]]))
    want = d.attend(k_lens=d.k_lens)
    assert ((short.double() - want.double()).abs() <= 2.0 ** -6 * want.double().abs() + 0.02).all()
    # a spoilt key inside the chunk
    q, m, labels = c.q_lens[0], c.k_lens[0], c.labels
    at = m - q + 150
    v = c.v.clone()
    v[at] = float("nan")
    c.c.append(c.k, v, c.lens, c.table, cu_rows=ints([0, m]))
    out = c.attend(k_lens=c.k_lens)
    pos = torch.arange(m - q, m, device="cuda")
    for h, kind in enumerate(labels):
        sees = at <= pos
        if kind:
            sees = sees & (pos - at < c.window)
        g = slice(h * (c.q.shape[1] // len(labels)), (h + 1) * (c.q.shape[1] // len(labels)))
        assert out[sees][:, g].isnan().all(), h
        x, y = out[~sees][:, g].double(), first[~sees][:, g].double()
        # (rows that are gone over again are summed in another order)
        assert ((x - y).abs() <= 2.0 ** -6 * y.abs() + 0.02).all(), h


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_items_of_several_sequences_in_parts(d, form):
    """Items that visit few tiles twice (8 bits: they are not written out), a sequence without keys among them."""
    c = Case([120, 119, 30, 120, 118], [9120, 8000, 0, 9119, 8500], 32, 8, d, [0, 1, 1, 0, 1, 1, 0, 1], 64, 512, 64, form, seed=d)
    first = c.attend(k_lens=c.k_lens).clone()
    c.matches("several sequences in parts")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # (without memory for states: clusters)
        c.c.attend(c.q, c.q_lens, c.lens, c.table, c.out, k_lens=c.k_lens)
    c.out.fill_(float("nan"))
    graph.replay()
    c.c.check()
    assert ((c.out.double() - first.double()).abs() <= 2.0 ** -6 * first.double().abs() + 0.02).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_without_any_key(d, form):
    """Zero, whatever the queries hold, in calls of many items and of one prompt."""
    c = Case([300 + 7 * (i % 5) for i in range(40)], [0] * 40, 16, 4, d, [0, 1, 0, 1], 4, 100, 64, form, seed=17)
    for _ in range(10):
        c.out.fill_(float("nan"))
        c.attend()
        assert (c.out == 0).all()
        c.out.fill_(float("nan"))
        c.c.prefill(c.q, c.k, c.v, c.q_lens, c.out, k_lens=c.k_lens)
        c.c.check()
        assert (c.out == 0).all()


def test_no_rows_and_no_sequences():
    c = Case([3, 0], [40, 20], 8, 2, 128, [0, 1], 4, 50, 16, "bf16")
    c.attend(k_lens=c.k_lens)
    c.matches("a sequence without rows")
    c.c.attend(c.q[:0], [0, 0], c.lens, c.table, c.out[:0])
    c.c.attend(c.q[:0], [], c.lens[:0], c.table[:0], c.out[:0])
    c.c.check()
