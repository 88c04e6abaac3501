"""A NaN in a query or in a key reaches the rows that it belongs to or that see it, and
no other, whichever CTAs share an item: a part of an item whose visible scores are all
NaN has no maximum (NaN is none), but it is not a part that saw no key."""

import pytest
import torch

from gpu_cases import ensure_lib
from paper_2608_06849_gb300 import aoh
from test_gpu_paged import prompt_inputs, sums

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


SHARED = [
    # q_lens, k_lens (None: the same), Hq, Hkv, d, labels, sink, window
    # clusters that split the keys of an item
    ([300], [3000], 32, 8, 64, [0] * 8, 0, 1),
    ([311], [2900], 16, 4, 128, [0, 0, 1, 0], 5, 900),
    ([40], [6000], 32, 8, 128, [0, 1] * 4, 9, 150),
    # items with one query tile, which both halves of a CTA's pipeline work on
    ([3, 1], [9000, 257], 4, 1, 128, [0], 0, 1),
    ([2, 11], [6300, 1], 16, 2, 64, [0, 1], 300, 3000),
    ([5], [4000], 2, 2, 64, [0, 1], 7, 90),
    # items that two CTAs share
    ([1100, 3], None, 4, 4, 128, [0, 1, 0, 1], 3, 50),
    ([1200], None, 4, 4, 64, [0, 1, 0, 0], 3, 700),
    # a CTA an item, and one pipeline through many
    ([600, 257], None, 7, 1, 128, [1], 200, 30),
    ([200 + 37 * (i % 9) for i in range(24)], None, 32, 8, 64, [0, 1] * 4, 9, 150),
]


def seen(pos, j, label, sink, window):
    return (j <= pos) & ((label == 0) | (j < sink) | (pos - j < window))


def run(case, q, k, v):
    q_lens, k_lens, hq, hkv, d, labels, sink, window = case
    pc = aoh.PagedCache(1, 16, hq, hkv, d, sink, window, labels, max_seqs=len(q_lens))
    out = torch.zeros((sum(q_lens), hq, d), dtype=torch.bfloat16, device="cuda")
    pc.prefill(q, k, v, q_lens, out, k_lens=k_lens)
    pc.check()
    return out


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_a_nan_query_row(case):
    q_lens, k_lens, hq, hkv, d, labels, sink, window = SHARED[case]
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=41)
    clean = run(SHARED[case], q, k, v)
    rows = sorted({0, sum(q_lens) // 2, sum(q_lens) - 1, min(128, sum(q_lens) - 1)})
    q[rows, :, 3] = float("nan")
    out = run(SHARED[case], q, k, v)
    # (a row before its sequence's first key sees none and gives zeros)
    pos = [m - n + i for n, m in zip(q_lens, q_lens if k_lens is None else k_lens) for i in range(n)]
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[[r for r in rows if pos[r] >= 0]] = True
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad], clean[~bad])


def spoilt_keys(kind, m, first):
    """Ranges of sequence positions, each for a call of its own: of m positions, rows from
    `first` on."""
    if kind == "first key":
        return [(0, 1)]
    # the first key of a tile, which the row at its position sees without another of the tile
    at = [j for j in range(0, m, 128) if j >= first][:10]
    if kind == "boundary key":
        return [(j, j + 1) for j in at]
    tiles = range(0, m, 128)
    return [(j, min(j + 128, m)) for j in tiles[::max(1, len(tiles) // 6)]] + [(0, m // 2)]


@pytest.mark.parametrize("kind", ["first key", "boundary key", "whole tiles"])
@pytest.mark.parametrize("case", range(len(SHARED)))
def test_nan_keys(case, kind):
    q_lens, k_lens, hq, hkv, d, labels, sink, window = SHARED[case]
    k_lens = q_lens if k_lens is None else k_lens
    q, k, v = prompt_inputs(q_lens, k_lens, hq, hkv, d, seed=43)
    clean = run(SHARED[case], q, k, v)
    b = 0  # the first sequence's keys
    pos = torch.arange(k_lens[b] - q_lens[b], k_lens[b], device="cuda")
    for j0, j1 in spoilt_keys(kind, k_lens[b], k_lens[b] - q_lens[b]):
        bad_k = k.clone()
        bad_k[sums(k_lens)[b] + j0:sums(k_lens)[b] + j1, :, 2] = float("nan")
        out = run(SHARED[case], q, bad_k, v)
        bad = torch.zeros_like(out, dtype=torch.bool)
        j = torch.arange(j0, j1, device="cuda")
        for h in range(hkv):
            sees = seen(pos[:, None], j[None, :], labels[h], sink, window).any(1)
            bad[:q_lens[b], h * (hq // hkv):(h + 1) * (hq // hkv)] = sees[:, None, None]
        assert torch.equal(torch.isnan(out), bad), (j0, j1)
        assert torch.equal(out[~bad], clean[~bad]), (j0, j1)


@pytest.mark.parametrize("d", [64, 128])
def test_a_cache_prefill_in_shared_items(d):
    """The same through a cache's prefill, whose items two CTAs share."""
    hq, hkv, T, labels, sink, window = 8, 4, 1100, [0, 1, 0, 1], 3, 50
    cache = aoh.Cache(1, hq, hkv, d, T, sink, window, labels)
    q, k, v = prompt_inputs([T], None, hq, hkv, d, seed=47)

    def prefill(q, k):
        out = torch.zeros_like(q)
        cache.reset()
        cache.prefill(q[None], k[None], v[None], out[None])
        cache.check()
        return out

    clean = prefill(q, k)
    bad_q = q.clone()
    bad_q[700, :, 1] = float("nan")
    out = prefill(bad_q, k)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[700] = True
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad], clean[~bad])
    pos = torch.arange(T, device="cuda")
    for j in (0, 128, 256, 512, 1024):
        bad_k = k.clone()
        bad_k[j, :, 0] = float("nan")
        out = prefill(q, bad_k)
        for h in range(hkv):
            bad[:, 2 * h:2 * h + 2] = seen(pos, j, labels[h], sink, window)[:, None, None]
        assert torch.equal(torch.isnan(out), bad), j
        assert torch.equal(out[~bad], clean[~bad]), j
    cache.close()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,hq,hkv", [([3000], 8, 2), ([30000, 20], 4, 2), ([700] * 40, 16, 4)])
def test_nan_keys_in_pages(form, d, lens, hq, hkv):
    """The paged decode: half of one head's keys, its first one, its last one."""
    page = 64
    per = [-(-n // page) for n in lens]
    table = torch.zeros((len(lens), max(per)), dtype=torch.int32)
    for b, n in enumerate(per):
        table[b, :n] = torch.arange(sum(per[:b]), sum(per[:b]) + n)
    pc = aoh.PagedCache(sum(per), page, hq, hkv, d, 0, 1, [0] * hkv, form=form, max_seqs=len(lens))
    table, t = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    cu = torch.tensor(sums(lens), dtype=torch.int32, device="cuda")
    _, k, v = prompt_inputs(lens, None, hkv, hkv, d, seed=53)
    q = prompt_inputs([len(lens)], None, hq, hkv, d, seed=59)[0]
    n = lens[0]
    for j0, j1 in ((0, n // 2), (n // 2, n), (0, 1), (n - 1, n)):
        bad = k.clone()
        bad[j0:j1, 0, 0] = float("nan")
        pc.append(bad, v, t, table, cu_rows=cu)
        for max_len in (0, 100):
            out = torch.zeros_like(q)
            pc.decode(q, t, table, out, max_len=max_len)
            pc.check()
            assert torch.isnan(out[0, :hq // hkv]).all(), (j0, j1)
            assert torch.isfinite(out[0, hq // hkv:]).all() and torch.isfinite(out[1:]).all(), (j0, j1)


@pytest.mark.parametrize("what,most", [("all values", 100), ("the first value", 35)])
def test_what_spoilt_values_cost(what, most):
    """Rows that are gone over again look at the keys that their tiles hide from them, and no
    longer than until all their numbers are NaN: with every V row NaN a call takes ten times as
    long as a clean one (a thousand times with every key gone over), with one that hides from
    nobody a dozen times (eighty)."""
    case = ([8192], None, 8, 2, 128, [0, 1], 4, 300)
    q, k, v = prompt_inputs(case[0], None, 8, 2, 128, seed=61)
    pc = aoh.PagedCache(1, 16, 8, 2, 128, 4, 300, case[5])
    out = torch.empty_like(q)

    def took(v):
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            pc.prefill(q, k, v, case[0], out)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    clean = took(v)
    assert torch.isfinite(out).all()
    spoilt = v.clone()
    spoilt[slice(None) if what == "all values" else 0] = float("nan") if what == "all values" else float("inf")
    assert took(spoilt) < most * clean
    pc.check()
