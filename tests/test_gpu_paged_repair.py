"""Parts of a few rows whose outputs a hidden V row has spoilt are computed again (include/aoh.h: a NaN or an
infinity reaches the rows that see it, and no other), whichever of a CTA's many items they are of and however long
their sequences: other items of the same CTA wait for none of it.

Tolerance: the rows are summed in another order and with weights of other bits than without the spoilt key, whose
weight the rows compared do not count: twice the rounding of each weight to 8 bits, 2^-8 of sum_j p_j |v_j| (at most
some 2 here, standard normal numbers), and of the output, 2^-9 of it, each: 2^-6 |o| + 0.02 covers both."""

import pytest
import torch

from gpu_cases import ensure_lib
from paper_2608_06849_gb300 import aoh

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def near(x, y):
    return ((x.double() - y.double()).abs() <= 2.0 ** -6 * y.double().abs() + 0.02).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, hkv", [(25, 64), (100, 64), (1100, 8)])
def test_any_item_of_a_run(n, hkv, d, form):
    """Up to 32 sequences, up to 1,024, more; more than 32 items a CTA in the latter two."""
    G, rows, page = 2, 4, 16
    q_lens = [1 + (3 * b) % rows for b in range(n)]
    k_lens = [q_lens[b] + 7 * (b % 29) for b in range(n)]
    need, width = -(-max(k_lens) // page), (1 << 17) // page
    c = aoh.PagedCache(n * need, page, G * hkv, hkv, d, 4, 30, [h % 2 for h in range(hkv)], form=form, max_seqs=n)
    c.pool.fill_(255)
    table, lens = torch.full((n, width), -1, dtype=torch.int32, device="cuda"), ints(k_lens)
    table[:, :need] = torch.randperm(n * need, device="cuda").int().view(n, need)
    ks, qs = [0], [0]
    for x, y in zip(k_lens, q_lens):
        ks.append(ks[-1] + x)
        qs.append(qs[-1] + y)
    k, v, q = randn((ks[-1], hkv, d), 1), randn((ks[-1], hkv, d), 2), randn((qs[-1], G * hkv, d), 3)
    out = torch.empty_like(q)
    hint = [1 << 17] * n  # lengths with which parts on the decode kernel are the choice
    c.append(k, v, lens, table, cu_rows=ints(ks))
    c.attend(q, q_lens, lens, table, out, k_lens=hint)
    c.check()
    clean = out.clone()
    assert torch.isfinite(clean).all()
    # one number of every third sequence's last V row, in every second head and another one each time
    last = torch.zeros(qs[-1], dtype=torch.bool, device="cuda")
    hit = torch.zeros((qs[-1], hkv), dtype=torch.bool, device="cuda")
    for b in range(0, n, 3):
        v[ks[b + 1] - 1, b % 2::2, (5 * b) % d] = float("nan")
        last[qs[b + 1] - 1] = True
        hit[qs[b + 1] - 1, b % 2::2] = True
    c.append(k, v, lens, table, cu_rows=ints(ks))
    for _ in range(3):
        out.fill_(0)
        c.attend(q, q_lens, lens, table, out, k_lens=hint)
        c.check()
        got, want = out.view(-1, hkv, G, d), clean.view(-1, hkv, G, d)
        assert got[hit].isnan().any(-1).all()
        assert near(got[~hit], want[~hit])


def test_a_long_sequence_holds_up_no_other_item():
    """Runs of four whole items of a million keys each: in one of them the first item's tokens see different parts
    of a last V row with an infinity. The keys of a column, one after the other, take longer than a wait of the
    kernel may."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    G, hkv, d, page, n_keys, n = 4, 1, 64, 128, 1 << 20, 4 * sms
    full = n_keys // page
    c = aoh.PagedCache(full + 1, page, G * hkv, hkv, d, 4, 30, [0], form="e4m3", max_seqs=n)
    k, v = randn((n_keys, hkv, d), 1), (randn((n_keys, hkv, d), 2).float() + 1).bfloat16()
    shared = torch.arange(full, dtype=torch.int32, device="cuda")
    c.append(k, v, ints([n_keys]), shared.view(1, -1), cu_rows=ints([0, n_keys]))
    at = 4 * (sms // 3)  # the first item of a run
    table = shared.repeat(n, 1)
    table[at, -1] = full  # its last page is its own
    q_lens = [4 if b == at else 1 for b in range(n)]
    q = randn((1, G, d), 3).repeat(sum(q_lens), 1, 1).contiguous()
    out = torch.empty_like(q)
    lens = ints([n_keys] * n)
    own = table[at:at + 1, -1:].contiguous()
    c.append(k[-page:], v[-page:], ints([page]), own, cu_rows=ints([0, page]))
    c.attend(q, q_lens, lens, table, out, k_lens=[n_keys] * n)
    c.check()
    clean = out.clone()
    v[-1, 0, 5] = float("inf")  # (a page holds it as NaN)
    c.append(k[-page:], v[-page:], ints([page]), own, cu_rows=ints([0, page]))
    out.fill_(0)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    c.attend(q, q_lens, lens, table, out, k_lens=[n_keys] * n)
    end.record()
    c.check()
    print(f"{start.elapsed_time(end):.0f} ms")
    others = torch.ones(sum(q_lens), dtype=torch.bool, device="cuda")
    others[at:at + 4] = False
    assert torch.equal(out[others], clean[others])
    # (a million numbers added one after the other, sums and weighted rows: at most 2^20 / 2 roundings of 2^-24 each)
    x, y = out[at:at + 4].double(), clean[at:at + 4].double()
    ok = (x - y).abs() <= 2.0 ** -4 * y.abs() + 0.02
    assert ok[:3].all() and ok[3, :, 6:].all() and ok[3, :, :5].all()
    assert not torch.isfinite(x[3, :, 5]).any()
