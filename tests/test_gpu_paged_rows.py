"""Rows of a call that no sequence has (buffers padded to a captured call's size, slots
of a step without a request)."""

import pytest
import torch

from gpu_cases import ensure_lib
from paper_2608_06849_gb300 import aoh
from test_gpu_paged import Pages, ints, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cu", [[0, 20, 37], [0, 37, 37], [3, 20, 37]])
def test_rows_behind_the_last_sequence(form, d, cu):
    """More rows than cu_rows gives out (and fewer than from its first on): what is nobody's is
    not written, although the last sequence's table goes on, and reported."""
    hkv, page, extra = 3, 16, 40
    lens = [30, 25] if cu[1] != 37 else [50, 25]
    p = Pages([n + 64 for n in lens], hkv, hkv, d, page, form, [0] * hkv, seed=d)
    n = cu[-1]
    k, v = randn((n + extra, hkv, d), 1), randn((n + extra, hkv, d), 2)
    outs = [torch.zeros((n + extra, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    first = ints([a - (cu[b + 1] - cu[b]) for b, a in enumerate(lens)])
    # the rows of the sequences alone
    p.cache.append(k[cu[0]:n], v[cu[0]:n], ints(lens), p.table, cu_rows=ints([c - cu[0] for c in cu]))
    p.cache.read(p.table, ints([c - cu[0] for c in cu]), outs[0][cu[0]:n], outs[1][cu[0]:n], first=first)
    p.cache.check()
    want = p.pool.clone()
    p.pool.fill_(255)
    for call in (lambda: p.cache.append(k, v, ints(lens), p.table, cu_rows=ints(cu)),
                 lambda: p.cache.read(p.table, ints(cu), outs[2], outs[3], first=first)):
        call()
        with pytest.raises(aoh.AohError) as e:
            p.cache.check()
        assert e.value.status == 1
        p.cache.check()
    assert torch.equal(p.pool, want)
    for a, b in ((0, 2), (1, 3)):
        assert torch.equal(outs[a][cu[0]:n], outs[b][cu[0]:n])


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_a_captured_step_with_idle_slots(form):
    """A slot without a request has length 0: nothing of it is written, its output is zeros,
    and no error is reported."""
    hq, hkv, d, page = 8, 2, 128, 16
    lens = [31, 15, 200, 5]
    p = Pages([n + 8 for n in lens], hq, hkv, d, page, form, [0, 1], 5, 40)
    p.fill(lens)
    k, v, q = randn((4, hkv, d), 1), randn((4, hkv, d), 2), randn((4, hq, d), 3)
    t, out = ints([n + 1 for n in lens]), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.cache.append(k, v, t, p.table)
        p.cache.decode(q, t, p.table, out)
    torch.cuda.current_stream().wait_stream(side)
    p.cache.check()
    want, pool = out.clone(), p.pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.append(k, v, t, p.table)
        p.cache.decode(q, t, p.table, out)
    for idle in (0, 3):
        t[idle] = 0
        out.fill_(float("nan"))
        graph.replay()
        p.cache.check()
        assert (out[idle] == 0).all()
        rest = [b for b in range(4) if t[b] > 0]
        assert torch.equal(out[rest], want[rest])
        assert torch.equal(p.pool, pool)
    # a negative length is an error all the same
    t[0] = -1
    graph.replay()
    with pytest.raises(aoh.AohError):
        p.cache.check()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_a_length_past_the_table(form):
    """Of a sequence whose length is past what its table holds no row is written, also not those
    that would still lie within; the other sequences' are."""
    hkv, d, page = 2, 64, 16
    lens, cu = [40, 20], ints([0, 5, 8])
    p = Pages([n + 16 for n in lens], hkv, hkv, d, page, form, [0] * hkv)
    table = ints([list(range(3)), [3, 4, 0]])
    k, v = randn((8, hkv, d), 1), randn((8, hkv, d), 2)
    p.cache.append(k[5:], v[5:], ints([20]), table[1:], cu_rows=ints([0, 3]))
    p.cache.check()
    want = p.pool.clone()
    p.pool.fill_(255)
    for past in (49, 51, 2 ** 31 - 1):
        p.cache.append(k, v, ints([past, 20]), table, cu_rows=cu)
        with pytest.raises(aoh.AohError):
            p.cache.check()
        assert torch.equal(p.pool, want)
    p.cache.append(k, v, ints([48, 20]), table, cu_rows=cu)  # to the last row of its table
    p.cache.check()
    assert not torch.equal(p.pool, want)
