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


BESIDE_A_CAPTURE = """
import sys
import torch
from paper_2608_06849_gb300 import aoh

FORM, ROWS, FRESH = sys.argv[1], int(sys.argv[2]), sys.argv[3] == "fresh"
HQ, HKV, D, PAGE, N = 32, 8, 128, 64, 20000
q = torch.randn(ROWS, HQ, D, device="cuda").bfloat16()
k, v = (torch.randn(N, HKV, D, device="cuda").bfloat16() for _ in range(2))
out = torch.empty_like(q)
pages = -(-N // PAGE)
table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
lens = torch.tensor([N], dtype=torch.int32, device="cuda")
cu = torch.tensor([0, N], dtype=torch.int32, device="cuda")


def handle():
    c = aoh.PagedCache(pages, PAGE, HQ, HKV, D, 16, 512, [0, 1] * (HKV // 2), form=FORM, max_seqs=1)
    c.append(k, v, lens, table, cu_rows=cu)
    return c


c = handle()
before = torch.cuda.mem_get_info()[0]
c.attend(q, [ROWS], lens, table, out, k_lens=[N])
torch.cuda.synchronize()
assert torch.cuda.mem_get_info()[0] < before, "the call took no memory"
want = out.clone()
if FRESH:
    c.close()
    c = handle()
other = torch.cuda.Stream()
a = torch.zeros(1, device="cuda")
torch.cuda.synchronize()
out.zero_()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a.add_(1)
    for _ in range(3):
        c.attend(q, [ROWS], lens, table, out, k_lens=[N], stream=other)
graph.replay()
torch.cuda.synchronize()
c.check()
assert a.item() == 1 and torch.equal(out, want)
print("both are right")
"""


def run(program, *args, says):
    ensure_lib()
    r = subprocess.run([sys.executable, "-c", program, *args], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and says in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def test_given_back_with_the_last_handle():
    run(PROGRAM, says="given back")


@pytest.mark.parametrize("pool", ["fresh", "kept"])
@pytest.mark.parametrize("form, rows", [("e4m3", 2048), ("bf16", 600)])
def test_taken_beside_a_capture(form, rows, pool):
    """A call that takes memory, on one stream, while another stream captures: neither ends the other, and the call
    gets its memory (the outputs are bit for bit those of the same call alone)."""
    run(BESIDE_A_CAPTURE, form, str(rows), pool, says="both are right")
