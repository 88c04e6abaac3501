"""NaN keys in one token's attention over a cache: where CTAs share an item and all keys
that one of them sees have a NaN score, its state has no maximum, and counts."""

import pytest
import torch

from gpu_cases import ensure_lib
from paper_2608_06849_gb300 import aoh
from paper_2608_06849_gb300.workloads import randn_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hq,Hkv,d,n", [(1, 8, 2, 64, 700), (40, 8, 2, 64, 700), (1, 14, 2, 64, 201), (1, 2, 2, 64, 30000),
                                          (1, 8, 2, 128, 700), (40, 8, 2, 128, 700), (1, 2, 2, 128, 30000)])
def test_nan_keys_reach_the_output(B, Hq, Hkv, d, n):
    ensure_lib()
    k, v = randn_bf16((B, n, Hkv, d), 11, "cuda"), randn_bf16((B, n, Hkv, d), 12, "cuda")
    q, kn, vn = (randn_bf16((B, h, d), 13 + h, "cuda") for h in (Hq, Hkv, Hkv))
    for j0, j1 in ((0, n // 2), (n // 2, n), (0, 1), (n - 1, n)):
        bad = k.clone()
        bad[:, j0:j1, 0] = float("nan")  # of one head: the others' outputs are numbers
        cache = aoh.Cache(B, Hq, Hkv, d, n + 1, 4, 60, [0] * Hkv)
        cache.prefill(None, bad, v)
        out = torch.empty_like(q)
        cache.decode_step(q, kn, vn, out)
        cache.check()
        cache.close()
        assert torch.isnan(out[:, :Hq // Hkv]).all(), (j0, j1)
        assert torch.isfinite(out[:, Hq // Hkv:]).all(), (j0, j1)
