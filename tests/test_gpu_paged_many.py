"""More work than one launch, or one block's shared memory, carries: prompts of more work
items than travel with a launch, by-value sequences and uploaded ones, and steps of more
sequences than have their lengths mirrored. Tolerances as in test_gpu_paged."""

import numpy as np
import pytest
import torch

from gpu_cases import assert_matches, ensure_lib, f64
from oracle import paged as opaged
from paper_2608_06849_gb300 import aoh
from test_gpu_paged import Pages, check_decode, ints, prompt_inputs, randn, sums

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _lib():
    ensure_lib()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_lens,hq,hkv,labels", [
    ([31000], 32, 8, [0] * 8),                              # 3,888 items of 122 tiles on average
    ([30000, 1500], 33, 11, [0] * 8 + [1, 0, 0]),           # with items of two tiles of a group's last head
    ([5800 + 7 * i for i in range(70)], 4, 2, [0, 0]),      # 70 sequences
])
def test_long_prompts_in_several_launches(d, q_lens, hq, hkv, labels):
    sink, window = 5, 300
    q, k, v = prompt_inputs(q_lens, None, hq, hkv, d, seed=7)
    pc = aoh.PagedCache(1, 16, hq, hkv, d, sink, window, labels, max_seqs=len(q_lens))
    out = torch.full_like(q, float("nan"))
    pc.prefill(q, k, v, q_lens, out)
    after = out.clone()  # ordered behind every launch
    pc.check()
    assert torch.equal(after, out)
    at = sums(q_lens)
    # rows of the heaviest items, which come first, and of the lightest, in the last launch
    for b in sorted({0, len(q_lens) // 2, len(q_lens) - 1}):
        n = q_lens[b]
        for r in (0, 1, 127, 128, 255, 300, n // 2, n - 129, n - 1):
            keys = slice(at[b], at[b] + r + 1)
            args, vb = (f64(q[at[b] + r:at[b] + r + 1]), f64(k[keys])), f64(v[keys])
            want = opaged.attend(*args, vb, labels, sink, window)
            mag = opaged.attend(*args, np.abs(vb), labels, sink, window)
            assert_matches(f64(out[at[b] + r:at[b] + r + 1]), want, f"row {r} of sequence {b}", mag=mag, abs_bounds=False)
    # every row, against the same prompt a KV head's queries at a time: few items, one launch
    for h in (0, hkv - 1):
        one = aoh.PagedCache(1, 16, hq // hkv, 1, d, sink, window, labels[h:h + 1], max_seqs=len(q_lens))
        heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
        alone = torch.empty_like(out[:, heads].contiguous())
        one.prefill(q[:, heads], k[:, h:h + 1], v[:, h:h + 1], q_lens, alone)
        one.check()
        assert torch.isfinite(alone).all() and (alone.float() - out[:, heads].float()).abs().max() <= 2.0 ** -5
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1024, 1025, 2100])
def test_a_step_of_many_sequences(form, n):
    hq, hkv, d, page, sink, window = 4, 2, 64, 16, 7, 60
    lens = [(37 * i + 11) % 190 for i in range(n)]
    lens[n // 2] = 3000
    p = Pages(lens, hq, hkv, d, page, form, [0, 1], sink, window)
    held = p.fill(lens)
    q = randn((n, hq, d), 3)
    for max_len in (0, 190):
        out = torch.full_like(q, float("nan"))
        p.cache.decode(q, ints(lens), p.table, out, max_len=max_len)
        p.cache.check()
        check_decode(out, q, held, [0, 1], sink, window, f"{n} sequences")
    # a length out of range is reported, and the others' outputs are as they were
    bad = list(lens)
    bad[5] = -3
    again = torch.empty_like(q)
    p.cache.decode(q, ints(bad), p.table, again)
    with pytest.raises(aoh.AohError):
        p.cache.check()
    rest = [b for b in range(n) if b != 5]
    assert (again[rest].float() - out[rest].float()).abs().max() <= 2.0 ** -5 * max(1.0, out.float().abs().max().item())
