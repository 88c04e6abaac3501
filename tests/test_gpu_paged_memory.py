"""The device memory that chunks over 8-bit pages take by themselves (written-out pages, states of items in
parts): kept between calls, given back with the device's last handle. In a process of its own: other
tests' handles would count."""

import subprocess
import sys

import pytest

from conftest import ROOT
from gpu_cases import ensure_lib

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch
from paper_2608_06849_gb300 import aoh

HQ, HKV, D, PAGE, N, ROWS = 32, 8, 128, 64, 60000, 2048
WRITTEN = 4 * D * HKV * (N // 128 * 128)  # bytes of the pages written out
q = torch.randn(ROWS, HQ, D, device="cuda").bfloat16()
k, v = (torch.randn(N, HKV, D, device="cuda").bfloat16() for _ in range(2))
out = torch.empty_like(q)
pages = -(-N // PAGE)
table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
lens = torch.tensor([N], dtype=torch.int32, device="cuda")
cu = torch.tensor([0, N], dtype=torch.int32, device="cuda")


def handle():
    c = aoh.PagedCache(pages, PAGE, HQ, HKV, D, 16, 512, [0] * HKV, form="e4m3", max_seqs=1)
    c.append(k, v, lens, table, cu_rows=cu)
    return c


def attend(c, times=1):
    for _ in range(times):
        c.attend(q, [ROWS], lens, table, out, k_lens=[N])


def free():
    return torch.cuda.mem_get_info()[0]


c, other = handle(), handle()
attend(c)  # every kernel's code is loaded now
torch.cuda.synchronize()
want = out.clone()
c.close()
other.close()
torch.cuda.synchronize()
for _ in range(2):
    c, other = handle(), handle()
    torch.cuda.synchronize()
    before = free()
    attend(c)
    torch.cuda.synchronize()
    assert before - free() >= WRITTEN, "the pages were not written out"
    c.close()
    torch.cuda.synchronize()
    assert before - free() >= WRITTEN // 2, "another handle lives, for which the memory is kept"
    # the last handle goes while its calls run
    attend(other, 5)
    other.close()
    torch.cuda.synchronize()
    assert free() >= before, f"{(before - free()) >> 20} MiB are kept without a handle"
    assert torch.equal(out, want)
    del c, other
print("given back")
"""


def test_given_back_with_the_last_handle():
    ensure_lib()
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "given back" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
