"""A server's attention over a paged cache, one layer: requests of different lengths are
admitted together, a long prompt comes in two chunks, and all of them then generate
tokens, one a step, in a captured graph.

    python examples/paged_serving.py [--form e4m3|bf16] [--steps N] [--rotary]

Queries, keys and values are random numbers in the place of a model's projections; with
--rotary the calls that write them to the pages normalise queries and keys and rotate them
by their positions. What a server keeps on the host is here a list of free pages and a page
list a request; the device sees a table and the lengths.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_06849_gb300 import aoh  # noqa: E402


class Server:
    """Requests' pages, and the calls of one attention layer. rotary: the layer's rope and its norm
    weights of queries and keys, (rope, q_norm, k_norm), or None: rows are used as they come."""

    def __init__(self, n_pages, page_size, n_q_heads, n_kv_heads, d_head, sink, window, labels, form, max_seqs, max_len,
                 rotary=None):
        self.cache = aoh.PagedCache(n_pages, page_size, n_q_heads, n_kv_heads, d_head, sink, window, labels, form=form,
                                    max_seqs=max_seqs)
        self.page_size, self.max_len, self.rotary = page_size, max_len, rotary
        self.free = list(range(n_pages))
        self.pages, self.lens = {}, {}
        self.table = torch.zeros((max_seqs, -(-max_len // page_size)), dtype=torch.int32, device="cuda")

    def grow(self, request, tokens):
        """Pages for `tokens` more tokens of a request."""
        pages = self.pages.setdefault(request, [])
        self.lens[request] = self.lens.get(request, 0) + tokens
        while len(pages) * self.page_size < self.lens[request]:
            pages.append(self.free.pop())

    def finish(self, request):
        self.free += self.pages.pop(request)
        del self.lens[request]

    def rows(self, requests):
        """Table rows and lengths of some requests, on the device."""
        host = torch.zeros((len(requests), self.table.shape[1]), dtype=torch.int32)
        for i, r in enumerate(requests):
            host[i, :len(self.pages[r])] = torch.tensor(self.pages[r], dtype=torch.int32)
        return host.cuda(), torch.tensor([self.lens[r] for r in requests], dtype=torch.int32, device="cuda")

    def append(self, q, k, v, lens, table, cu=None):
        """New rows written to the pages; the queries that attend."""
        if self.rotary is None:
            self.cache.append(k, v, lens, table, cu_rows=cu)
            return q
        rope, q_norm, k_norm = self.rotary
        turned = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        self.cache.append_rotated(rope, q, k, v, lens, table, turned, cu_rows=cu, q_norm=q_norm, k_norm=k_norm)
        return turned

    def prompts(self, requests, tokens, q, k, v):
        """`tokens[i]` more rows of requests[i]'s prompt, packed: their keys and values written, and
        their attention. Rows that continue a prompt see what its pages hold."""
        before = [self.lens.get(r, 0) for r in requests]
        for r, n in zip(requests, tokens):
            self.grow(r, n)
        table, lens = self.rows(requests)
        cu = torch.tensor([0] + list(tokens), dtype=torch.int32, device="cuda").cumsum(0, dtype=torch.int32)
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        q = self.append(q, k, v, lens, table, cu)
        if any(before) or self.rotary is not None:
            self.cache.attend(q, list(tokens), lens, table, out, k_lens=[self.lens[r] for r in requests])
        else:
            self.cache.prefill(q, k, v, list(tokens), out)
        return out

    def capture(self, requests, steps, q, k, v):
        """A graph of one token step of these requests, with pages for `steps` of them."""
        for r in requests:
            self.grow(r, steps)
            self.lens[r] -= steps
        self.step_table, self.step_lens = self.rows(requests)
        out = torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step_lens.add_(1)
            turned = self.append(q, k, v, self.step_lens, self.step_table)
            self.cache.decode(turned, self.step_lens, self.step_table, out, max_len=self.max_len)
        return graph, out


def run(form="e4m3", steps=16, prompts=(700, 45, 1300), chunk=512, n_q_heads=32, n_kv_heads=8, d_head=128, sink=64,
        window=512, page_size=64, seed=0, watch=None, rotary=None):
    """Serve the prompts and `steps` tokens; `watch(kind, requests, tokens, q, k, v, out)` sees
    every call's inputs and outputs. rotary: as Server has it."""
    watch = watch or (lambda *a: None)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def tokens(n):
        rows = torch.randn((n, n_q_heads + 2 * n_kv_heads, d_head), generator=g, device="cuda").bfloat16()
        return rows[:, :n_q_heads], rows[:, n_q_heads:n_q_heads + n_kv_heads], rows[:, n_q_heads + n_kv_heads:]

    labels = [h % 2 for h in range(n_kv_heads)]
    max_len = max(prompts) + steps
    pages = sum(-(-(n + steps) // page_size) for n in prompts)
    s = Server(pages, page_size, n_q_heads, n_kv_heads, d_head, sink, window, labels, form, len(prompts), max_len, rotary)
    # all prompts at once, at most `chunk` tokens of each a call
    left, requests = list(prompts), list(range(len(prompts)))
    while any(left):
        now = [r for r in requests if left[r] > 0]
        count = [min(left[r], chunk) for r in now]
        q, k, v = tokens(sum(count))
        out = s.prompts(now, count, q, k, v)
        watch("prompt", now, count, q, k, v, out)
        for r, n in zip(now, count):
            left[r] -= n
    # then a token of each a step
    q, k, v = (x.contiguous() for x in tokens(len(requests)))
    graph, out = s.capture(requests, steps, q, k, v)
    for _ in range(steps):
        for x, y in zip((q, k, v), tokens(len(requests))):
            x.copy_(y)
        graph.replay()
        watch("token", requests, [1] * len(requests), q, k, v, out)
    s.cache.check()
    for r in requests:
        s.finish(r)
    assert len(s.free) == pages
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--form", choices=("e4m3", "bf16"), default="e4m3")
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--rotary", action="store_true")
    a = ap.parse_args()
    ones = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    last = run(form=a.form, steps=a.steps, rotary=(aoh.Rope(128, base=500000.0), ones, ones) if a.rotary else None)
    torch.cuda.synchronize()
    print(f"served 3 prompts and {a.steps} tokens each; last outputs have rms {last.float().pow(2).mean().sqrt():.3f}")
