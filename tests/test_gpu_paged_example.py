"""The paged serving example, each call's outputs against the 64-bit definition over what
the pages hold."""

import importlib.util
import os

import numpy as np
import pytest

from gpu_cases import assert_matches, ensure_lib, f64
from oracle import paged as opaged

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

    def held(x):
        return x if form == "bf16" else opaged.decode(*opaged.encode(x))

    def watch(kind, requests, tokens, q, k, v, out):
        q, k, v, out = f64(q), f64(k), f64(v), f64(out)
        first = not past
        at = 0
        for r, n in zip(requests, tokens):
            rows = slice(at, at + n)
            at += n
            # a first call's prompts attend to their keys as they are, later ones to the pages
            use = (lambda x: x) if kind == "prompt" and first else held
            old = past.get(r, (np.zeros((0, 2, d)), np.zeros((0, 2, d))))
            kk, vv = (np.concatenate([a, use(b[rows])]) for a, b in zip(old, (k, v)))
            want = opaged.attend(q[rows], kk, vv, labels, sink, window)
            mag = opaged.attend(q[rows], kk, np.abs(vv), labels, sink, window)
            assert_matches(out[rows], want, f"{kind} of request {r}", mag=mag, abs_bounds=False)
            past[r] = tuple(np.concatenate([a, held(b[rows])]) for a, b in zip(old, (k, v)))

    example.run(form=form, steps=5, prompts=(300, 20, 450), chunk=200, n_q_heads=8, n_kv_heads=2, d_head=d, sink=sink,
                window=window, page_size=32, watch=watch)
    assert [len(past[r][0]) for r in range(3)] == [305, 25, 455]
