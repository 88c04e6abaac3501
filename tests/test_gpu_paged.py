"""The paged operators against their 64-bit definitions (oracle.paged): packed prompts,
rows written to pages and read back, and attention of one token over pages.

Tolerance of attention outputs: rounding each softmax weight to at least 8 significant
bits moves an output by at most 2^-9 * sum_j p_j |v_j| (``mag``, the definition run on
|v|), storing it as bf16 by 2^-9 |o|; twice both plus 1e-4 is allowed
(gpu_cases.assert_matches). What pages hold is compared bit by bit."""

import numpy as np
import pytest
import torch

from gpu_cases import assert_matches, ensure_lib, f64
from oracle import paged as opaged
from paper_2608_06849_gb300 import aoh

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


def randn(shape, seed, scale=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    if scale is not None:
        x *= torch.exp2(scale * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    return x.bfloat16()


def ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def sums(xs):
    return np.concatenate([[0], np.cumsum(xs)]).tolist()


# ------------------------------------------------------------------ prompts

PROMPTS = [
    # q_lens, k_lens (None: the same), Hq, Hkv, d, labels, sink, window
    ([5], None, 2, 1, 64, [0], 0, 1),
    ([1], None, 4, 4, 128, [0, 1, 0, 1], 0, 1),
    ([1, 128, 0, 129, 127, 300], None, 8, 2, 128, [0, 1], 4, 40),
    ([77, 1, 513, 64], None, 8, 2, 64, [1, 0], 0, 130),
    ([600, 257], None, 7, 1, 128, [1], 200, 30),
    ([1300], None, 14, 2, 128, [0, 1], 128, 256),
    ([90, 1, 200], [400, 1000, 200], 6, 2, 128, [0, 1], 16, 100),
    ([33, 5], [1290, 129], 16, 1, 64, [0], 0, 1),
    ([300, 7, 130], [10, 0, 131], 4, 2, 128, [0, 1], 2, 3),
    ([9, 260], [0, 0], 4, 2, 64, [0, 1], 2, 3),
    ([3 + 5 * (i % 7) for i in range(70)], None, 4, 2, 64, [0, 1], 8, 9),
    ([140 + 31 * (i % 5) for i in range(40)], None, 24, 8, 128, [0, 1] * 4, 8, 100),
    ([40] * 130, [60] * 130, 32, 8, 64, [0] * 8, 0, 1),
    # few rows of many heads: heads fold into the tiles; after long prefixes the keys are split
    ([17, 3, 1], [3000, 2999, 1], 32, 8, 64, [0, 1] * 4, 10, 500),
    ([33, 20], [2500, 900], 7, 1, 128, [0], 0, 1),
    ([5, 100, 26], [2049, 10, 1500], 10, 2, 128, [0, 1], 100, 300),
    ([16, 9], [1900, 1281], 16, 1, 128, [0], 0, 1),
    ([9] * 30, [9 + 50 * (i % 4) for i in range(30)], 24, 2, 64, [1, 0], 3, 70),
    ([30 - i % 25 for i in range(70)], None, 40, 8, 128, [0, 1] * 4, 2, 11),
    ([70], [1111], 6, 2, 128, [0, 1], 128, 129),
    ([1, 1, 1, 1], [5000, 100, 1, 640], 8, 1, 128, [0], 0, 1),
    # one query tile an item, its keys shared by both halves of the pipeline: small clusters, ...
    ([1 + i % 16 for i in range(60)], [1500 + 64 * i for i in range(60)], 24, 3, 64, [0, 1, 0], 5, 1100),
    # ... and clusters of 16, with one query tile an item and with two
    ([3, 1], [9000, 257], 4, 1, 128, [0], 0, 1),
    ([100], [7003], 4, 2, 128, [0, 0], 0, 1),
    ([2, 11], [6300, 1], 16, 2, 64, [0, 1], 300, 3000),
    # a query head a KV head: few rows and long ones after long prefixes
    ([5], [4000], 2, 2, 64, [0, 1], 7, 90),
    ([300, 40], [3333, 2600], 3, 3, 128, [0, 1, 0], 0, 1000),
    # clusters whose size is no power of two
    ([300], [3000], 32, 8, 64, [0] * 8, 0, 1),
    ([311], [2900], 16, 4, 128, [0, 0, 1, 0], 5, 900),
    ([140, 150], [2000, 1700], 5, 5, 128, [0, 1, 0, 0, 0], 5, 900),
    # heads of 64: items that two CTAs share, long ones, and many with several tiles
    ([1200], None, 4, 4, 64, [0, 1, 0, 0], 3, 700),
    ([1700, 900], [1900, 900], 16, 8, 64, [0, 1] * 4, 3, 700),
    ([200 + 37 * (i % 9) for i in range(24)], None, 32, 8, 64, [0, 1] * 4, 9, 150),
]


def prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=0, fused=False):
    nq, nk = sum(q_lens), sum(q_lens if k_lens is None else k_lens)
    q, k, v = randn((nq, hq, d), seed), randn((nk, hkv, d), seed + 1), randn((nk, hkv, d), seed + 2)
    if fused:
        qkv = torch.cat([q, k, v], 1)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    return q, k, v


def check_prompts(out, q, k, v, q_lens, k_lens, labels, sink, window, what):
    k_lens = q_lens if k_lens is None else k_lens
    qs, ks = sums(q_lens), sums(k_lens)
    q, k, v, out = f64(q), f64(k), f64(v), f64(out)
    for b in range(len(q_lens)):
        if q_lens[b] == 0:
            continue
        args = (q[qs[b]:qs[b + 1]], k[ks[b]:ks[b + 1]])
        vb = v[ks[b]:ks[b + 1]]
        want = opaged.attend(*args, vb, labels, sink, window)
        mag = opaged.attend(*args, np.abs(vb), labels, sink, window)
        assert_matches(out[qs[b]:qs[b + 1]], want, f"{what}, sequence {b}", mag=mag, abs_bounds=False)


@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(case):
    q_lens, k_lens, hq, hkv, d, labels, sink, window = PROMPTS[case]
    fused = k_lens is None and case % 2 == 1
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=10 * case, fused=fused)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, sink, window, labels, max_seqs=len(q_lens))
    out = torch.full((sum(q_lens), hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
    pc.check()
    check_prompts(out, q, k, v, q_lens, k_lens, labels, sink, window, f"prompts {case}")


def test_many_work_items_in_several_launches():
    """More items than travel with one launch: the launches' rows are all written."""
    q_lens = [128] * 130
    hq, hkv, d = 64, 32, 64
    q, k, v = prompt_inputs(q_lens, None, hq, hkv, d)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, 0, 1, [0] * hkv, max_seqs=len(q_lens))
    out = torch.full_like(q, float("nan"))
    pc.prefill(q, k, v, q_lens, out)
    after = out.clone()  # ordered behind every launch
    pc.check()
    assert torch.equal(after, out)
    for b in (0, 59, 60, 61, 119, 120, 129):
        at = slice(128 * b, 128 * (b + 1))
        check_prompts(out[at], q[at], k[at], v[at], [128], None, [0] * hkv, 0, 1, f"sequence {b}")
    assert torch.isfinite(out.float()).all()


def test_prompts_do_not_see_their_neighbours():
    """NaN in one sequence's q, k and v leaves the others' outputs as they are."""
    q_lens, hq, hkv, d, labels = [70, 200, 33], 8, 2, 128, [0, 1]
    q, k, v = prompt_inputs(q_lens, None, hq, hkv, d, seed=5)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, 4, 50, labels)
    out = torch.empty_like(q)
    pc.prefill(q, k, v, q_lens, out)
    for x in (q, k, v):
        x[70:270] = float("nan")
    again = torch.empty_like(q)
    pc.prefill(q, k, v, q_lens, again)
    pc.check()
    keep = list(range(70)) + list(range(270, 303))
    assert torch.equal(out[keep], again[keep])


SPOILT = [PROMPTS[i] for i in (2, 3, 5, 6, 10, 11, 13, 14, 18, 20, 21, 23)]
SPOILT.append(([1100, 3], None, 4, 4, 128, [0, 1, 0, 1], 3, 50))  # items that two CTAs share


@pytest.mark.parametrize("what", ["nan in k and v", "inf in v"])
@pytest.mark.parametrize("case", range(len(SPOILT)))
def test_prompts_do_not_see_hidden_keys(case, what):
    """A NaN or an infinity in a key reaches the rows that see the key, and no other: neither
    rows before it nor those whose window it has left."""
    q_lens, k_lens, hq, hkv, d, labels, sink, window = SPOILT[case]
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=3)
    clean = (k.clone(), v.clone())
    k_lens = q_lens if k_lens is None else k_lens
    ks, spoilt = sums(k_lens), []
    for b, m in enumerate(k_lens):
        first = max(m - q_lens[b], 0)
        # among a sequence's rows, and at its end
        spoilt.append(sorted({first + (m - first) // 2, m - 1}) if m > first + 1 else [])
        for j in spoilt[b]:
            at = ks[b] + j
            if what == "inf in v":
                v[at, :, 5] = float("inf")
                clean[1][at, :, 5] = 0
            else:
                k[at, :, 2] = float("nan")
                v[at, :, 1::2] = float("nan")
                clean[0][at], clean[1][at] = 0, 0
    pc = aoh.PagedCache(1, 16, hq, hkv, d, sink, window, labels, max_seqs=len(q_lens))
    out = torch.zeros((sum(q_lens), hq, d), dtype=torch.bfloat16, device="cuda")
    pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
    pc.check()
    # what sees a spoilt key is not finite, and left out of the comparison
    want_bad = torch.zeros_like(out, dtype=torch.bool)
    row = 0
    for b, n in enumerate(q_lens):
        pos = torch.arange(k_lens[b] - n, k_lens[b], device="cuda")
        for j in spoilt[b]:
            for h in range(hkv):
                sees = (j <= pos) & ((labels[h] == 0) | (j < sink) | (pos - j < window))
                heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                if what == "inf in v":
                    want_bad[row:row + n, heads, 5] |= sees[:, None]
                else:
                    want_bad[row:row + n, heads] |= sees[:, None, None]
        row += n
    assert torch.equal(~torch.isfinite(out), want_bad)
    if what == "inf in v":  # infinite weights do not mix signs here
        assert (out[want_bad] == float("inf")).all()
    again = torch.zeros_like(out)
    pc.prefill(q, *clean, q_lens, again, k_lens=k_lens)
    pc.check()
    rows = ~want_bad.any(-1).any(-1)
    out[want_bad] = 0
    again[want_bad] = 0
    ref, got = f64(again[rows]), f64(out[rows])
    # the same sums, once with weights rounded to bf16 and once not
    assert np.abs(ref - got).max(initial=0) <= 2.0 ** -6 * max(1.0, np.abs(ref).max(initial=0))
    for b, r in [(b, r) for b, n in enumerate(q_lens) for r in range(0, n, max(1, n // 5))][:40]:
        at, m = sums(q_lens)[b] + r, k_lens[b] - q_lens[b] + r + 1
        if rows[at] and m > 0:
            keys = slice(ks[b], ks[b] + m)
            args, vb = (f64(q[at:at + 1]), f64(clean[0][keys])), f64(clean[1][keys])
            want = opaged.attend(*args, vb, labels, sink, window)
            mag = opaged.attend(*args, np.abs(vb), labels, sink, window)
            assert_matches(f64(out[at:at + 1]), want, f"row {r} of sequence {b}", mag=mag, abs_bounds=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["many", "long", "split"])
def test_prompts_come_out_alike_every_time(d, kind):
    """The same call with its tensors in and out of the cache: bit for bit the same."""
    hq, hkv = 32, 8
    q_lens, k_lens = {"many": ([200 + 37 * (i % 9) for i in range(24)], None), "long": ([2500], None),
                      "split": ([40], [6000])}[kind]
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=9)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, 9, 150, [0, 1] * 4, max_seqs=len(q_lens))
    want = torch.empty_like(q)
    pc.prefill(q, k, v, q_lens, want, k_lens=k_lens)
    flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(60):
        if i % 2:
            flush.fill_(i)
        out = torch.full_like(q, float("nan"))
        pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
        bad += (out != want).any().long()
    pc.check()
    assert bad.item() == 0


@pytest.mark.parametrize("g,hkv", [(3, 8), (7, 4)])
def test_short_prompts_after_nans_in_shared_memory(g, hkv):
    """Rows of a tile that are nobody's, whose contents are whatever lay there, cost
    nothing: the call takes as long after one whose tensors are all NaN."""
    d, q_lens = 64, [15 + i % 20 for i in range(100)]
    q, k, v = prompt_inputs(q_lens, None, g * hkv, hkv, d)
    pc = aoh.PagedCache(1, 16, g * hkv, hkv, d, 8, 30, [i % 2 for i in range(hkv)], max_seqs=len(q_lens))
    out = torch.empty_like(q)

    def timed():
        best = float("inf")
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda._sleep(1000000)
            a.record()
            pc.prefill(q, k, v, q_lens, out)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    timed()
    before = timed()
    want = out.clone()
    n = 1500
    bad = torch.full((n, g * hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pc.prefill(bad, bad[:, :hkv], bad[:, :hkv], [n], torch.empty_like(bad))
    after = timed()
    pc.check()
    assert torch.equal(out, want)
    assert after < 3 * before + 0.02, (before, after)


@pytest.mark.parametrize("case", [2, 6, 10, 13])
def test_prompts_in_a_graph(case):
    """A captured call, by-value sequences and uploaded ones, replays with new inputs."""
    q_lens, k_lens, hq, hkv, d, labels, sink, window = PROMPTS[case]
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=1)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, sink, window, labels, max_seqs=len(q_lens))
    out = torch.empty_like(q)
    pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
    q2, k2, v2 = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=7)
    want = torch.empty_like(q)
    pc.prefill(q2, k2, v2, q_lens, want, k_lens=k_lens)
    for x, y in ((q, q2), (k, k2), (v, v2)):
        x.copy_(y)
    out.fill_(float("nan"))
    graph.replay()
    pc.check()
    assert torch.equal(out, want)


# ------------------------------------------------------------------ pages

class Pages:
    """A pool of NaN bytes, tables that deal its pages in a mixed order, and what the
    pages should hold."""

    def __init__(self, lens, hq, hkv, d, page, form, labels, sink=0, window=1, seed=0, extra=3):
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + extra
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(self.n_pages, generator=g, dtype=torch.int32)
        self.table = torch.full((len(lens), max(1, max(need)) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.page, self.form, self.hkv, self.d = page, form, hkv, d
        self.host_table = self.table.numpy().copy()
        self.table = self.table.cuda()
        cfg = aoh.make_paged_config(hq, hkv, d, page, self.n_pages, form, max(1, len(lens)), sink, window)
        self.pool = torch.full((aoh.aoh_paged_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
        self.cache = aoh.PagedCache(self.n_pages, page, hq, hkv, d, sink, window, labels, form=form,
                                    max_seqs=max(1, len(lens)), pool=self.pool)
        self.expect = np.full(self.pool.shape, 255, dtype=np.uint8)

    def put(self, b, first, k, v):
        """Rows k, v [n, Hkv, d] (float64 of bf16 numbers) at positions first .. in ``expect``."""
        n, p = k.shape[0], self.page
        pos = np.arange(first, first + n)
        page, row = self.host_table[b, pos // p], pos % p
        numbers = self.n_pages * 2 * self.hkv * p * self.d
        for sel, x in ((0, k), (1, v)):
            if self.form == "bf16":
                data = self.expect.view(np.uint16).reshape(self.n_pages, 2, self.hkv, p, self.d)
                bits = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
                for i in range(n):
                    data[page[i], sel, :, row[i]] = bits[i]
            else:
                data = self.expect[:numbers].reshape(self.n_pages, 2, self.hkv, p, self.d)
                powers = self.expect[numbers:].view(np.int8).reshape(self.n_pages, self.hkv, 2, p)
                codes, e = opaged.encode(x)
                for i in range(n):
                    data[page[i], sel, :, row[i]] = codes[i]
                    powers[page[i], :, sel, row[i]] = e[i]

    def held(self, x):
        """What a row holds of x."""
        return x if self.form == "bf16" else opaged.decode(*opaged.encode(x))

    def fill(self, lens, seed=0):
        """Write a sequence's tokens through append; K, V as the pages hold them."""
        k, v = randn((sum(lens), self.hkv, self.d), seed + 1), randn((sum(lens), self.hkv, self.d), seed + 2, scale=2.0)
        self.cache.append(k, v, ints(lens), self.table, cu_rows=ints(sums(lens)))
        self.cache.check()
        at = sums(lens)
        return [(self.held(f64(k[a:b])), self.held(f64(v[a:b]))) for a, b in zip(at, at[1:])]


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_and_read(form, d, page):
    rows, before, hkv = [37, 1, 0, 130, 64], [0, 5, 9, 17, 64], 3
    lens = [a + b for a, b in zip(rows, before)]
    p = Pages(lens, hkv, hkv, d, page, form, [0] * hkv, seed=page)
    k, v = randn((sum(rows), hkv, d), 1, scale=6.0), randn((sum(rows), hkv, d), 2)
    k[3] = 0
    k[4, 1, 3:] = 0
    v[5, 0, 7] = float("inf")
    v[6, 2, 9] = float("nan")
    v[7, 2, 1] = -float("inf")
    k[8] *= 2.0 ** 125
    k[9] *= 2.0 ** -100
    v[10, 0] = 464.0
    kv = torch.cat([k, torch.zeros_like(k), v], 1)  # strided rows
    at = sums(rows)
    p.cache.append(kv[:, :hkv], kv[:, 2 * hkv:], ints(lens), p.table, cu_rows=ints(at))
    p.cache.check()
    got = p.pool.cpu().numpy()
    fk, fv = f64(k), f64(v)
    for b in range(len(rows)):
        p.put(b, before[b], fk[at[b]:at[b + 1]], fv[at[b]:at[b + 1]])
    if form == "bf16":
        # NaN payloads may differ
        g, e = (torch.from_numpy(x.view(np.int16).copy()).view(torch.bfloat16).float().numpy() for x in (got, p.expect))
        assert np.array_equal(g, e, equal_nan=True)
    else:
        numbers = p.n_pages * 2 * hkv * page * d
        sign = np.where((got[:numbers] & 127) == 127, 127, got[:numbers])  # NaN has no sign
        want = np.where((p.expect[:numbers] & 127) == 127, 127, p.expect[:numbers])
        assert np.array_equal(sign, want)
        assert np.array_equal(got[numbers:], p.expect[numbers:])
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    p.cache.read(p.table, ints(at), k_out, v_out, first=ints(before))
    p.cache.check()
    for out, x in ((k_out, fk), (v_out, fv)):
        want = torch.from_numpy(p.held(x)).to(torch.bfloat16)
        assert np.array_equal(f64(out), want.double().numpy(), equal_nan=True)


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_append_and_read_one_row_each(form):
    n, hkv, d, page = 9, 8, 128, 16
    lens = [1 + 5 * i for i in range(n)]
    p = Pages(lens, hkv, hkv, d, page, form, [0] * hkv)
    k, v = randn((n, hkv, d), 1), randn((n, hkv, d), 2)
    p.cache.append(k, v, ints(lens), p.table)
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    p.cache.read(p.table, None, k_out, v_out, first=ints([x - 1 for x in lens]))
    p.cache.check()
    assert np.array_equal(f64(k_out), p.held(f64(k)))
    assert np.array_equal(f64(v_out), p.held(f64(v)))


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_aligned_to_16_bytes_alone(form, d):
    lens, hkv, page = [50, 3], 3, 16
    p = Pages(lens, hkv, hkv, d, page, form, [0] * hkv)
    n, width = sum(lens), hkv * d
    raw = randn((2 * n + 1, width + 8), 1)
    rows = [raw.as_strided((n, hkv, d), (width + 8, d, 1), 8 + i * n * (width + 8)) for i in range(2)]
    assert rows[0].data_ptr() % 32 == 16
    cu = ints(sums(lens))
    p.cache.append(rows[0], rows[1], ints(lens), p.table, cu_rows=cu)
    outs = [torch.empty(n * width + 8, dtype=torch.bfloat16, device="cuda")[8:].view(n, hkv, d) for _ in range(2)]
    p.cache.read(p.table, cu, *outs)
    p.cache.check()
    for out, x in zip(outs, rows):
        assert np.array_equal(f64(out), p.held(f64(x)))


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_append_many_rows(form):
    """Enough rows for blocks of several."""
    lens, hkv, d, page = [3001, 1, 2500], 2, 64, 32
    p = Pages(lens, hkv, hkv, d, page, form, [0] * hkv)
    k, v = randn((sum(lens), hkv, d), 1, scale=3.0), randn((sum(lens), hkv, d), 2)
    cu = ints(sums(lens))
    p.cache.append(k, v, ints(lens), p.table, cu_rows=cu)
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    p.cache.read(p.table, cu, k_out, v_out)
    p.cache.check()
    assert np.array_equal(f64(k_out), p.held(f64(k)))
    assert np.array_equal(f64(v_out), p.held(f64(v)))


# ------------------------------------------------------------------ decode

DECODE = [
    # lens, Hq, Hkv, d, labels, sink, window
    ([1], 1, 1, 128, [0], 0, 1),
    ([0, 1, 2, 15, 16, 17], 4, 2, 128, [0, 1], 3, 5),
    ([127, 128, 129, 255, 256, 257], 8, 2, 64, [1, 0], 20, 100),
    ([700, 0, 33], 7, 1, 128, [0], 0, 1),
    ([1500, 511], 16, 1, 128, [0], 0, 1),
    ([900, 513, 512], 32, 2, 64, [1, 0], 1, 77),
    ([2000], 28, 4, 128, [0, 1, 0, 1], 128, 300),
    ([5000, 1, 300], 6, 2, 64, [0, 1], 0, 64),
    ([3, 4100], 5, 1, 128, [1], 130, 1000),
    ([600], 3, 1, 64, [1], 0, 1),
    ([97 * i % 400 for i in range(50)], 16, 8, 128, [0, 1] * 4, 7, 60),
    ([20000, 9000, 30], 8, 2, 128, [0, 1], 16, 500),
]


def check_decode(out, q, held, labels, sink, window, what):
    q, out = f64(q), f64(out)
    for b, (k, v) in enumerate(held):
        if k.shape[0] == 0:
            assert (out[b] == 0).all(), what
            continue
        want = opaged.attend(q[b:b + 1], k, v, labels, sink, window)
        mag = opaged.attend(q[b:b + 1], k, np.abs(v), labels, sink, window)
        assert_matches(out[b:b + 1], want, f"{what}, sequence {b}", mag=mag, abs_bounds=False)


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(case, form):
    lens, hq, hkv, d, labels, sink, window = DECODE[case]
    page = [16, 32, 64, 128][(case + (form == "bf16")) % 4]
    p = Pages(lens, hq, hkv, d, page, form, labels, sink, window, seed=case)
    held = p.fill(lens, seed=100 * case)
    wide = randn((len(lens), hq + 3, d), 7)
    q = wide[:, :hq]
    out = torch.full((len(lens), hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    p.cache.decode(q, ints(lens), p.table, out)
    p.cache.check()
    check_decode(out, q, held, labels, sink, window, f"decode {case} {form}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 4, 9])
def test_decode_whatever_the_bound(form, d, hkv):
    """Both splits of the work (max_len chooses) on the same step: long and short
    sequences, one without a token, one of a single one."""
    lens, hq, sink, window = [3000, 1, 0, 517, 130], 7 * hkv, 30, 200
    labels = [i % 2 for i in range(hkv)]
    p = Pages(lens, hq, hkv, d, 32, form, labels, sink, window)
    held = p.fill(lens, seed=hkv)
    q = randn((len(lens), hq, d), 3)
    for max_len in (0, 1, 200, 100000):
        out = torch.full_like(q, float("nan"))
        p.cache.decode(q, ints(lens), p.table, out, max_len=max_len)
        p.cache.check()
        check_decode(out, q, held, labels, sink, window, f"bound {max_len}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [9, 16])
def test_decode_with_many_heads_whatever_the_bound(form, d, g):
    """As above, with as many query heads a KV head as there can be."""
    lens, hkv, sink, window = [2900, 0, 1, 700], 2, 30, 200
    labels = [0, 1]
    p = Pages(lens, g * hkv, hkv, d, 16, form, labels, sink, window)
    held = p.fill(lens, seed=g)
    q = randn((len(lens), g * hkv, d), 4)
    for max_len in (0, 1, 200, 100000):
        out = torch.full_like(q, float("nan"))
        p.cache.decode(q, ints(lens), p.table, out, max_len=max_len)
        p.cache.check()
        check_decode(out, q, held, labels, sink, window, f"bound {max_len}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_with_a_heavy_first_key(form, d):
    """An attention sink with a small value, far above the other keys: their sum still
    counts (its weight is e^6 to e^12 of each of theirs)."""
    lens, hq, hkv = [9000, 2300], 8, 2
    p = Pages(lens, hq, hkv, d, 32, form, [0, 0])
    k, v = randn((sum(lens), hkv, d), 1), randn((sum(lens), hkv, d), 2)
    q = randn((2, hq, d), 3)
    at = sums(lens)
    for b in range(2):
        for h in range(hkv):
            k[at[b], h] = 4.0 * q[b, h * (hq // hkv)]
            v[at[b], h] *= 2.0 ** -6
    p.cache.append(k, v, ints(lens), p.table, cu_rows=ints(at))
    out = torch.empty_like(q)
    p.cache.decode(q, ints(lens), p.table, out)
    p.cache.check()
    held = [(p.held(f64(k[a:b])), p.held(f64(v[a:b]))) for a, b in zip(at, at[1:])]
    check_decode(out, q, held, [0, 0], 0, 1, f"sink {form} {d}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_decode_does_not_see_hidden_rows(form):
    """Positions outside a streaming head's sinks and window may hold NaN."""
    lens, hq, hkv, d, sink, window = [1000, 300], 8, 2, 128, 10, 50
    p = Pages(lens, hq, hkv, d, 64, form, [1, 1], sink, window)
    k, v = randn((sum(lens), hkv, d), 1), randn((sum(lens), hkv, d), 2)
    at = sums(lens)
    for b, n in enumerate(lens):
        for x in (k, v):
            x[at[b] + sink:at[b] + n - window] = float("nan")
    p.cache.append(k, v, ints(lens), p.table, cu_rows=ints(at))
    q = randn((2, hq, d), 3)
    out = torch.empty_like(q)
    p.cache.decode(q, ints(lens), p.table, out)
    p.cache.check()
    held = [(p.held(f64(k[a:b])), p.held(f64(v[a:b]))) for a, b in zip(at, at[1:])]
    for b in range(2):
        for x in held[b]:
            x[sink:lens[b] - window] = 0
    check_decode(out, q, held, [1, 1], sink, window, f"hidden rows {form}")


def test_decode_twice_and_on_another_stream():
    """The workspace is left clean, and a call runs on the stream it is given."""
    lens, hq, hkv, d = [5000, 60, 2000], 8, 2, 128
    p = Pages(lens, hq, hkv, d, 64, "e4m3", [0, 1], 4, 300)
    held = p.fill(lens)
    q, t = randn((3, hq, d), 3), ints(lens)
    outs = [torch.empty_like(q) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p.cache.decode(q, t, p.table, outs[0], stream=side)
    with torch.cuda.stream(side):
        p.cache.decode(q, t, p.table, outs[1])
        p.cache.decode(q, t, p.table, outs[2])
    p.cache.check(stream=side)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    check_decode(outs[0], q, held, [0, 1], 4, 300, "side stream")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_steps_in_a_graph(form):
    """A captured step (append, then decode) sees the lengths and tables of its replay."""
    hq, hkv, d, page = 8, 2, 128, 16
    lens = [31, 15, 200]
    p = Pages([n + 40 for n in lens], hq, hkv, d, page, form, [0, 1], 5, 40)
    k, v = randn((sum(lens), hkv, d), 1), randn((sum(lens), hkv, d), 2)
    at = sums(lens)
    p.cache.append(k, v, ints(lens), p.table, cu_rows=ints(at))
    held = [(p.held(f64(k[a:b])), p.held(f64(v[a:b]))) for a, b in zip(at, at[1:])]
    q, kn, vn = randn((3, hq, d), 3), randn((3, hkv, d), 4), randn((3, hkv, d), 5)
    t = ints([n + 1 for n in lens])
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.cache.append(kn, vn, t, p.table)
        p.cache.decode(q, t, p.table, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.append(kn, vn, t, p.table)
        p.cache.decode(q, t, p.table, out)
        t.add_(1)
    for step in range(20):
        kn.copy_(randn((3, hkv, d), 50 + step))
        vn.copy_(randn((3, hkv, d), 90 + step))
        q.copy_(randn((3, hq, d), 130 + step))
        graph.replay()
        p.cache.check()
        for b in range(3):
            held[b] = tuple(np.concatenate([x, p.held(f64(new[b:b + 1]))]) for x, new in zip(held[b], (kn, vn)))
        if step in (0, 1, 18, 19):
            check_decode(out, q, held, [0, 1], 5, 40, f"step {step}")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_a_prompt_continued_from_its_pages(form):
    """Prefixes read back from the pages, then the next rows: what a whole prompt over
    the held numbers gives."""
    hq, hkv, d, labels, sink, window = 8, 2, 128, [0, 1], 20, 150
    before, rows = [300, 45], [130, 77]
    p = Pages([a + b for a, b in zip(before, rows)], hq, hkv, d, 32, form, labels, sink, window)
    total = [a + b for a, b in zip(before, rows)]
    k, v, q = randn((sum(total), hkv, d), 1), randn((sum(total), hkv, d), 2), randn((sum(rows), hq, d), 3)
    p.cache.append(k, v, ints(total), p.table, cu_rows=ints(sums(total)))
    k_held, v_held = torch.empty_like(k), torch.empty_like(v)
    p.cache.read(p.table, ints(sums(total)), k_held, v_held)
    out = torch.empty_like(q)
    p.cache.prefill(q, k_held, v_held, rows, out, k_lens=total)
    p.cache.check()
    assert np.array_equal(f64(k_held), p.held(f64(k)))
    check_prompts(out, q, k_held, v_held, rows, total, labels, sink, window, "continued")


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_offsets_past_32_bits(form):
    """Pages at the end of a pool of more than 2^32 elements."""
    hq, hkv, d, page, lens = 8, 8, 128, 128, [300, 5]
    n_pages = 2 ** 32 // (2 * hkv * page * d) + 700
    pc = aoh.PagedCache(n_pages, page, hq, hkv, d, 0, 1, [0] * hkv, form=form, max_seqs=2)
    assert pc.nbytes > 2 ** 32
    table = ints([[n_pages - 1, n_pages - 3, n_pages - 2], [n_pages - 600, 0, 1]])
    k, v, q = randn((sum(lens), hkv, d), 1), randn((sum(lens), hkv, d), 2), randn((2, hq, d), 3)
    at = sums(lens)
    pc.append(k, v, ints(lens), table, cu_rows=ints(at))
    held = [torch.empty_like(k), torch.empty_like(v)]
    pc.read(table, ints(at), *held)
    out = torch.empty_like(q)
    pc.decode(q, ints(lens), table, out)
    pc.check()
    want = [f64(k), f64(v)] if form == "bf16" else [opaged.decode(*opaged.encode(f64(x))) for x in (k, v)]
    for x, w in zip(held, want):
        assert np.array_equal(f64(x), w)
    check_decode(out, q, [tuple(w[a:b] for w in want) for a, b in zip(at, at[1:])], [0] * hkv, 0, 1, "far pages")


def test_out_of_range_tables_are_reported():
    """A page or a length out of range touches nothing outside the pool and is
    reported once."""
    lens, hq, hkv, d = [40, 20], 4, 2, 128
    for form in ("bf16", "e4m3"):
        p = Pages(lens, hq, hkv, d, 16, form, [0, 1], 2, 64)
        p.fill(lens)
        before = p.pool.clone()
        k, q = randn((2, hkv, d), 1), randn((2, hq, d), 2)
        out = torch.empty_like(q)
        for bad in (-1, p.n_pages, 2 ** 31 - 1, -2 ** 31):
            table = p.table.clone()
            table[0, 2] = bad
            for call in (lambda: p.cache.append(k, k, ints([40, 1000]), table),
                         lambda: p.cache.decode(q, ints(lens), table, out)):
                call()
                with pytest.raises(aoh.AohError) as e:
                    p.cache.check()
                assert e.value.status == 1
                p.cache.check()
            assert torch.equal(before, p.pool)
        for bad in (-5, 16 * p.table.shape[1] + 1, 2 ** 31 - 1):
            p.cache.decode(q, ints([bad, 20]), p.table, out)
            with pytest.raises(aoh.AohError):
                p.cache.check()
        p.cache.decode(q, ints(lens), p.table, out)
        p.cache.check()


def test_calls_without_rows():
    p = Pages([20], 4, 2, 64, 16, "bf16", [0, 0])
    z, table = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), p.table[:0]
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    none = ints([])
    p.cache.append(z, z, none, table)
    p.cache.append(z, z, ints([20]), p.table, cu_rows=ints([0, 0]))
    p.cache.read(p.table, ints([0, 0]), z, torch.empty_like(z))
    p.cache.decode(q, none, table, torch.empty_like(q))
    p.cache.prefill(q, z, z, [], torch.empty_like(q))
    p.cache.prefill(q, z, z, [0, 0][:1], torch.empty_like(q))
    p.cache.check()
