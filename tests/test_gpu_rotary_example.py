"""The paged serving example with norms and rotation: rotated appends, chunks over the pages and
captured token steps together, each call's outputs against the 64-bit definition.

The definition is given queries and keys as the kernels round them (bf16, or codes). A number whose
32-bit rotation lies within 2^-20 of a border may be rounded the other way: one in 2^12 of a query's, by
2^-7 of it, and one in 2^16 of a key's codes, by 2^-3. With rows of size 1.1 a score moves by about 1.2 * 2^-7 /
sqrt(d) then, 0.0012, or that of one key by 0.02; the second is one weight among some hundred, so that
an output moves by at most 2 * 0.0012 of sum_j p_j |v_j| (``mag``). The usual 2^-8 of it is doubled: 0.0039 more.
"""

import importlib.util
import os

import numpy as np
import pytest
import torch

from gpu_cases import assert_matches, bf16_round, ensure_lib, f64
from oracle import paged as opaged
from oracle import rotary as orot
from paper_2608_06849_gb300 import aoh

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_serving(form, d):
    ensure_lib()
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    sink, window, labels, past = 10, 100, [0, 1], {}
    g = torch.Generator(device="cuda").manual_seed(1)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    freqs = orot.frequencies(d // 2, 1e4)
    rope = aoh.Rope(inv_freq=freqs, scale=1.1)

    def turned(x, w, pos):
        return orot.rotate(orot.norm(f64(x), f64(w), 1e-6), pos, freqs, scale=1.1)

    def held(x):
        return bf16_round(x) if form == "bf16" else opaged.decode(*opaged.encode(x))

    def watch(kind, requests, tokens, q, k, v, out):
        out, at = f64(out), 0
        for r, n in zip(requests, tokens):
            rows = slice(at, at + n)
            at += n
            old = past.get(r, (np.zeros((0, 2, d)), np.zeros((0, 2, d))))
            pos = np.arange(len(old[0]), len(old[0]) + n)
            qq = bf16_round(turned(q[rows], wq, pos))
            kk = np.concatenate([old[0], held(turned(k[rows], wk, pos))])
            vv = np.concatenate([old[1], held(f64(v[rows]))])
            past[r] = kk, vv
            want = opaged.attend(qq, kk, vv, labels, sink, window)
            mag = 2 * opaged.attend(qq, kk, np.abs(vv), labels, sink, window)
            assert_matches(out[rows], want, f"{kind} of request {r}", mag=mag, abs_bounds=False)

    example.run(form=form, steps=5, prompts=(300, 20, 450), chunk=200, n_q_heads=8, n_kv_heads=2, d_head=d, sink=sink,
                window=window, page_size=32, watch=watch, rotary=(rope, wq, wk))
    assert [len(past[r][0]) for r in range(3)] == [305, 25, 455]
