"""Memory and tensors of a GPU that is not the handle's are refused before the library is
called (it takes bare pointers, and its handles belong to the current device). No GPU:
tensors that say where they are, and a current device that is set here."""

import pytest
import torch

from paper_2608_06849_gb300 import aoh
from paper_2608_06849_gb300 import build as aoh_build


class On:
    """A tensor that says it is on a GPU."""

    is_cuda = True

    def __init__(self, t, index=0):
        self.t, self.index = t, index
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture(autouse=True)
def two_gpus(monkeypatch):
    aoh_build.build()
    aoh.load()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    # what gets this far was not refused
    for name in ("aoh_paged_init", "aoh_cache_init"):
        monkeypatch.setattr(aoh, name, lambda *a: pytest.fail("reached the library"))


def paged(**kw):
    return aoh.PagedCache(4, 16, 8, 2, 64, 0, 1, [0, 0], **kw)


def test_a_pool_on_another_gpu():
    pool = torch.zeros(4 * 2 * 2 * 16 * 64 * 2, dtype=torch.uint8)
    for kw in (dict(pool=On(pool, 1)), dict(pool=pool), dict(device="cuda:1"), dict(device=1), dict(device="cpu")):
        with pytest.raises(ValueError, match="current device, cuda:0"):
            paged(**kw)


@pytest.mark.parametrize("current,device", [(0, "cuda:1"), (0, 1), (1, 0), (0, "cpu")])
def test_a_cache_on_another_gpu(monkeypatch, current, device):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    with pytest.raises(ValueError, match=f"current device, cuda:{current}"):
        aoh.Cache(1, 8, 2, 64, 16, 0, 1, [0, 0], device=device)


def test_tensors_on_another_gpu(monkeypatch):
    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    monkeypatch.setattr(aoh, "aoh_paged_init", lambda *a: None)
    c = paged(pool=On(torch.zeros(4 * 2 * 2 * 16 * 64 * 2, dtype=torch.uint8)))
    monkeypatch.setattr(aoh, "_lib", Lib())
    monkeypatch.setattr(c, "_stream", lambda stream: 0)

    def bf(*shape):
        return On(torch.zeros(*shape, dtype=torch.bfloat16))

    def ints(*shape):
        return On(torch.zeros(*shape, dtype=torch.int32))

    def each(f, *tensors):
        """All on the pool's GPU, then one after the other elsewhere."""
        before = len(calls)
        f(*tensors)
        assert len(calls) == before + 1
        for i in range(len(tensors)):
            there = [On(t.t, 1) if i == j else t for j, t in enumerate(tensors)]
            with pytest.raises(ValueError, match="cuda:1, the pool on cuda:0"):
                f(*there)
        assert len(calls) == before + 1

    k, q, table = bf(3, 2, 64), bf(3, 8, 64), ints(3, 9)
    each(lambda q, k, v, out: c.prefill(q, k, v, [1, 2], out), q, k, k, q)
    each(lambda k, v, lens, table: c.append(k, v, lens, table), k, k, ints(3), table)
    each(lambda k, v, lens, table, cu: c.append(k, v, lens, table, cu_rows=cu), k, k, ints(3), table, ints(4))
    each(lambda table, k, v: c.read(table, None, k, v), table, k, k)
    each(lambda table, cu, k, v, first: c.read(table, cu, k, v, first=first), table, ints(4), k, k, ints(3))
    each(lambda q, lens, table, out: c.decode(q, lens, table, out), q, ints(3), table, q)
    c.handle = None
