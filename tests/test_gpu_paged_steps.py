"""Calls as a server makes them, one after the other or captured: single tokens by the attention of chunks and by the
decode, slots whose request ends between replays, a prompt's chunk beside many single tokens.

Tolerances: against the 64-bit definition as in test_gpu_paged_attend.py."""

import numpy as np
import pytest
import torch

from gpu_cases import assert_matches, ensure_lib, f64
from oracle import paged as opaged
from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh
from test_gpu_paged_attend import Case, held, ints, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_by_either_call(form, d):
    """Both are held to the definition, from both sides."""
    lens = [1, 700, 33, 2048, 129, 0, 16]
    c = Case([1] * 7, lens, 8, 2, d, [0, 1], 10, 100, 16, form, seed=3)
    out = c.attend(k_lens=lens).clone()
    c.matches("attend", [0, 1, 2, 3, 4, 6])
    c.out.fill_(float("nan"))
    c.c.decode(c.q, c.lens, c.table, c.out)
    c.c.check()
    c.matches("decode", [0, 1, 2, 3, 4, 6])
    assert (out[5] == 0).all() and (c.out[5] == 0).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("drafted", [1, 3])
def test_a_slot_that_ends_between_replays(form, drafted):
    """A graph of append and attend over two slots. The second one's request ends: its length becomes 0 and its table
    names no page. Its rows give zeros, its queries and its former pages stay, the other slot goes on; a step of several
    tokens a slot reports the rows that have no place, one of a token a slot none (include/aoh.h: cu_rows)."""
    hq, hkv, d, page, S, W = 8, 2, 128, 16, 4, 40
    rope, freqs = aoh.Rope(d), orot.frequencies(d, 1e4)
    c = aoh.PagedCache(40, page, hq, hkv, d, S, W, [0, 1], form=form, max_seqs=2)
    n = 2 * drafted
    table, lens = ints(np.arange(40).reshape(2, 20)), ints([0, 0])
    cu = None if drafted == 1 else ints([0, drafted, n])
    q, k, v = randn((n, hq, d), 0), randn((n, hkv, d), 1), randn((n, hkv, d), 2)
    turned, out, step = torch.empty_like(q), torch.empty_like(q), ints([drafted, drafted])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(step)
        c.append_rotated(rope, q, k, v, lens, table, turned, cu_rows=cu)
        c.attend(turned, [drafted, drafted], lens, table, out)
    past = [[np.zeros((0, hkv, d))] * 2 for _ in range(2)]

    def replay(i, live):
        for j, x in enumerate((q, k, v)):
            x.copy_(randn(tuple(x.shape), 100 * i + j))
        out.fill_(float("nan"))
        graph.replay()
        for b in range(live):
            rows = slice(b * drafted, (b + 1) * drafted)
            pos = np.arange(i * drafted, (i + 1) * drafted)
            kk = orot.rotate(f64(k[rows]), pos, freqs)
            kk = f64(torch.from_numpy(kk).bfloat16()) if form == "bf16" else opaged.decode(*opaged.encode(kk))
            past[b] = [np.concatenate([past[b][0], kk]), np.concatenate([past[b][1], held(v[rows], form)])]
            want = opaged.attend(f64(turned[rows]), *past[b], [0, 1], S, W)
            mag = opaged.attend(f64(turned[rows]), past[b][0], np.abs(past[b][1]), [0, 1], S, W)
            assert_matches(f64(out[rows]), want, f"step {i}, slot {b}", mag=mag, abs_bounds=False)

    for i in range(12):
        replay(i, 2)
    c.check()
    pages = table[1].clone()
    before = c.pool.clone()
    lens[1] = 0
    step[1] = 0
    table[1] = -1
    queries = turned[drafted:].clone()
    for i in range(12, 15):
        replay(i, 1)
        assert (out[drafted:] == 0).all() and torch.equal(turned[drafted:], queries)
        if drafted == 1:
            c.check()
        else:
            with pytest.raises(aoh.AohError, match="out of range"):
                c.check()
    bytes_of_page = 2 * hkv * page * d * (1 if form == "e4m3" else 2)
    for p in pages.tolist():
        at = slice(p * bytes_of_page, (p + 1) * bytes_of_page)
        assert torch.equal(c.pool.view(torch.uint8)[at], before.view(torch.uint8)[at])


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_a_chunk_beside_many_single_tokens(form):
    """Whatever the host takes the lengths to be: right, too short, absent."""
    q_lens = [1] * 20 + [700] + [1] * 43
    k_lens = [1 + 61 * i for i in range(20)] + [2900] + [900 + 7 * i for i in range(43)]
    c = Case(q_lens, k_lens, 16, 4, 128, [0, 1, 0, 0], 20, 300, 32, form, seed=4)
    for hint in (k_lens, [x // 3 for x in k_lens], None):
        c.out.fill_(float("nan"))
        c.attend(k_lens=hint)
        c.matches(f"hint {hint and hint[:3]}")


def test_outputs_over_queries_are_refused():
    """(A spoilt value in reach would have rows computed again from queries that are no longer there.)"""
    n, hq, d = 6, 8, 64
    c = Case([2, 4], [40, 50], hq, 2, d, [0, 1], 4, 30, 16, "bf16")
    size = n * hq * d
    buffer = torch.zeros(3 * size, dtype=torch.bfloat16, device="cuda")
    q = buffer[size:2 * size].view(n, hq, d)
    q.copy_(c.q)
    for at in (size, size + 8, 8, 2 * size - 8):
        with pytest.raises(aoh.AohError, match="must not overlap"):
            c.c.attend(q, c.q_lens, c.lens, c.table, buffer[at:at + size].view(n, hq, d))
    want = c.attend()
    for at in (0, 2 * size):
        out = buffer[at:at + size].view(n, hq, d)
        c.c.attend(q, c.q_lens, c.lens, c.table, out)
        assert torch.equal(out, want)
    # a slice of a fused projection: the last row ends with its own heads
    fused = torch.zeros(n * 2 * hq * d + size, dtype=torch.bfloat16, device="cuda")
    q = fused[:n * 2 * hq * d].view(n, 2 * hq, d)[:, :hq]
    q.copy_(c.q)
    end = (2 * n - 1) * hq * d
    for at, ok in ((end, True), (end - 8, False)):
        out = fused[at:at + size].view(n, hq, d)
        if ok:
            c.c.attend(q, c.q_lens, c.lens, c.table, out)
            assert torch.equal(out, want)
        else:
            with pytest.raises(aoh.AohError, match="must not overlap"):
                c.c.attend(q, c.q_lens, c.lens, c.table, out)
    c.c.check()
