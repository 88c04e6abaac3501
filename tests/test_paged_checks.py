"""Refusals of the paged cache: the binding's checks of tensors (before any pointer reaches
the library) and the library's checks of configurations and arguments. No GPU: a
PagedCache object is assembled without a pool, and right CPU tensors get as far as being
refused as CPU tensors."""

import ctypes

import pytest
import torch

from paper_2608_06849_gb300 import aoh
from paper_2608_06849_gb300 import build as aoh_build


@pytest.fixture(scope="module")
def lib():
    aoh_build.build()
    return aoh.load()


def cache(hq=8, hkv=2, d=64, max_seqs=4):
    c = object.__new__(aoh.PagedCache)
    c.handle, c.max_seqs = None, max_seqs
    c.n_q_heads, c.n_kv_heads, c.d_head = hq, hkv, d
    return c


class Cuda:
    """A tensor that says it is on a GPU."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def bf(*shape):
    return Cuda(torch.zeros(*shape, dtype=torch.bfloat16))


def ints(*shape):
    return Cuda(torch.zeros(*shape, dtype=torch.int32))


def refused(match, f, *args, **kw):
    with pytest.raises(ValueError, match=match):
        f(*args, **kw)


def test_prefill_tensors(lib):
    c = cache()
    q, k, out = bf(10, 8, 64), bf(10, 2, 64), bf(10, 8, 64)
    refused("^q has shape", c.prefill, bf(10, 7, 64), k, k, [10], out)
    refused("^q has shape", c.prefill, bf(10, 8 * 64), k, k, [10], out)
    refused("^k has shape", c.prefill, q, bf(10, 2, 128), k, [10], out)
    refused("^out has shape", c.prefill, q, k, k, [10], bf(9, 8, 64))
    refused("say otherwise", c.prefill, q, k, k, [9], out)
    refused("say otherwise", c.prefill, q, k, k, [10], out, k_lens=[11])
    refused("say otherwise", c.prefill, q, k, bf(11, 2, 64), [10], out)
    refused("one length a sequence", c.prefill, q, k, k, [2] * 5, out)
    refused("one length a sequence", c.prefill, q, k, k, [5, 5], out, k_lens=[10])
    refused("CUDA tensor", c.prefill, torch.zeros(10, 8, 64, dtype=torch.bfloat16), k, k, [10], out)
    refused("bfloat16", c.prefill, Cuda(torch.zeros(10, 8, 64)), k, k, [10], out)
    refused("dense rows", c.prefill, Cuda(torch.zeros(10, 64, 8, dtype=torch.bfloat16).transpose(1, 2)), k, k, [10], out)
    refused("dense rows", c.prefill, Cuda(torch.zeros(1, 8, 64, dtype=torch.bfloat16).expand(10, 8, 64)), k, k, [10], out)
    refused("contiguous", c.prefill, q, k, k, [10], Cuda(torch.zeros(10, 16, 64, dtype=torch.bfloat16)[:, :8]))


def test_append_and_read_tensors(lib):
    c = cache()
    k, lens, table = bf(3, 2, 64), ints(3), ints(3, 9)
    refused("for 4 sequences", c.append, k, k, ints(4), ints(4, 9))
    refused("^k and v hold", c.append, k, bf(2, 2, 64), lens, table)
    refused("^lens has shape", c.append, k, k, ints(2), table)
    refused("^lens must be", c.append, k, k, Cuda(torch.zeros(3, dtype=torch.int64)), table)
    refused("^table has shape", c.append, k, k, lens, ints(27))
    refused("^table has shape", c.append, k, k, ints(5), ints(5, 9))
    refused("^table must be", c.append, k, k, lens, Cuda(torch.zeros(9, 3, dtype=torch.int32).t()))
    refused("^cu_rows has shape", c.append, k, k, lens, table, cu_rows=ints(3))
    refused("^k_out has shape", c.read, table, None, bf(3, 2, 32), k)
    refused("^v_out has shape", c.read, table, None, k, bf(2, 2, 64))
    refused("rows for 3 sequences", c.read, table, None, bf(4, 2, 64), bf(4, 2, 64))
    refused("^first has shape", c.read, table, ints(4), k, k, first=ints(4))


def test_decode_tensors(lib):
    c = cache()
    q, lens, table, out = bf(3, 8, 64), ints(3), ints(3, 9), bf(3, 8, 64)
    refused("q holds 2 rows", c.decode, bf(2, 8, 64), lens, table, out)
    refused("^q has shape", c.decode, bf(3, 2, 64), lens, table, out)
    refused("^out has shape", c.decode, q, lens, table, bf(4, 8, 64))
    refused("^lens has shape", c.decode, q, ints(3, 1), table, out)


GOOD = dict(n_q_heads=8, n_kv_heads=2, d_head=64, page_size=16, n_pages=10, form="e4m3", max_seqs=4, sink=0, window=1)


def test_configurations(lib):
    assert aoh.aoh_paged_bytes(aoh.make_paged_config(**GOOD)) == 10 * 2 * 2 * 16 * (64 + 1)
    assert aoh.aoh_paged_bytes(aoh.make_paged_config(**dict(GOOD, form="bf16"))) == 10 * 2 * 2 * 16 * 64 * 2
    for bad in (dict(n_q_heads=7), dict(n_kv_heads=0), dict(n_kv_heads=65, n_q_heads=65), dict(n_q_heads=34),
                dict(d_head=96), dict(page_size=24), dict(page_size=256), dict(n_pages=0), dict(n_pages=2 ** 29),
                dict(max_seqs=0), dict(max_seqs=65536), dict(sink=-1), dict(window=0), dict(window=2 ** 30 + 1)):
        with pytest.raises(aoh.AohError):
            aoh.aoh_paged_bytes(aoh.make_paged_config(**dict(GOOD, **bad)))
    with pytest.raises(ValueError, match="form"):
        aoh.make_paged_config(**dict(GOOD, form="int8"))
    cfg = aoh.make_paged_config(**GOOD)
    cfg.form = 2
    with pytest.raises(aoh.AohError):
        aoh.aoh_paged_bytes(cfg)


def test_init_refuses_on_the_host(lib):
    cfg, h = aoh.make_paged_config(**GOOD), ctypes.c_void_p()
    good, bad = (ctypes.c_uint8 * 2)(0, 1), (ctypes.c_uint8 * 2)(0, 2)
    n = aoh.aoh_paged_bytes(cfg)
    pool = ctypes.c_void_p(1 << 20)
    assert lib.aoh_paged_init(ctypes.byref(cfg), good, pool, n, None) == 1
    assert lib.aoh_paged_init(ctypes.byref(cfg), None, pool, n, ctypes.byref(h)) == 1
    assert lib.aoh_paged_init(ctypes.byref(cfg), bad, pool, n, ctypes.byref(h)) == 1
    assert "head_labels[1]" in lib.aoh_last_error().decode()
    assert lib.aoh_paged_init(ctypes.byref(cfg), good, None, n, ctypes.byref(h)) == 1
    assert lib.aoh_paged_init(ctypes.byref(cfg), good, ctypes.c_void_p((1 << 20) + 16), n, ctypes.byref(h)) == 1
    assert lib.aoh_paged_init(ctypes.byref(cfg), good, pool, n - 1, ctypes.byref(h)) == 2
    assert h.value is None
    with pytest.raises(ValueError, match="labels"):
        aoh.aoh_paged_init(cfg, [0], torch.zeros(8, dtype=torch.uint8))


def test_calls_without_a_handle(lib):
    p = ctypes.c_void_p(1 << 20)
    one = (ctypes.c_int32 * 1)(1)
    assert lib.aoh_paged_append(None, p, p, 128, 128, None, p, 1, 1, p, 1, None) == 1
    assert lib.aoh_paged_read(None, None, None, 1, 1, p, 1, p, p, None) == 1
    assert lib.aoh_paged_decode(None, p, 512, p, 1, 0, p, 1, p, None) == 1
    assert lib.aoh_paged_prefill(None, p, p, p, 512, 128, 128, one, None, 1, p, None) == 1
    assert lib.aoh_paged_check(None, None) == 1
    lib.aoh_paged_destroy(None)
