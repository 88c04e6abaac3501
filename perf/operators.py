"""The paged serving operators, as measurable cases.

A server holds the keys and values of many requests in pages of a fixed number
of tokens and serves them in one call each:

  prompt   causal attention over prompts of different lengths packed one behind
           the other; with more keys than queries, the rows that continue a
           prompt whose earlier keys are known
  cache    a call's new keys and values written to the pages (as bf16, or as
           8-bit numbers with a power of two for each row), and read back
  decode   attention of one new token of every sequence over the pages

Retrieval KV heads see every earlier position, streaming heads the first `sink`
positions and the last `window`. Shapes are those of the repository's workloads
(28/4 and 32/8 heads of 128, 32/8 and 8/2 heads of 64) and generic ones.

`own` false: the operators in elementary torch operations, in 32 bits. `own`
true: the calls of ``paper_2608_06849_gb300.aoh.PagedCache``.

A pool of pages holds [pages][K, V][kv heads][page tokens][d], and behind it, with
8-bit numbers (e4m3), the powers of two as int8 [pages][kv heads][K, V][page
tokens]: a stored number x of a row with power e stands for x * 2^e. e is the
least one with which the row's largest finite number is at most 448, in [-80, 120].
"""

import math
import random

import torch

own = False

E_MIN, E_MAX = -80, 120


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a few short questions of a small model: latency
        dict(name="prompt_short_d64", kind="prompt", seqs=5, low=1, high=190, prefix=0, q_heads=8, kv_heads=2,
             d_head=64, sink=16, window=128, streaming=1, fused=False),
        # a scheduler's batch of prompts, as slices of the fused projection's output
        dict(name="prompt_b16_ragged", kind="prompt", seqs=16, low=101, high=2999, prefix=0, q_heads=32, kv_heads=8,
             d_head=128, sink=64, window=512, streaming=4, fused=True),
        # one long prompt: the largest pass
        dict(name="prompt_32k", kind="prompt", seqs=1, low=32768, high=32768, prefix=0, q_heads=28, kv_heads=4,
             d_head=128, sink=128, window=2048, streaming=2, fused=False),
        # later chunks of four prompts, behind prefixes read back from the pages
        dict(name="prompt_b4_continued", kind="prompt", seqs=4, low=700, high=2048, prefix=8001, q_heads=32, kv_heads=8,
             d_head=128, sink=64, window=2048, streaming=0, fused=False),
        # one token of each of 64 sequences, written and read: latency
        dict(name="cache_step_b64", kind="cache", seqs=64, low=1, high=1, prefix=4096, kv_heads=8, d_head=128,
             page=64, form="e4m3"),
        # the batch of prompts above, into 8 bits and back
        dict(name="cache_b16_ragged", kind="cache", seqs=16, low=101, high=2999, prefix=0, kv_heads=8, d_head=128,
             page=64, form="e4m3"),
        # a long prompt of 64-wide heads into small bf16 pages, continuing in the middle of one
        dict(name="cache_32k_d64", kind="cache", seqs=1, low=32768, high=32768, prefix=4097, kv_heads=8, d_head=64,
             page=16, form="bf16"),
        # batch-1 chat at a short context: latency
        dict(name="decode_b1_4k", kind="decode", seqs=1, low=4096, high=4096, q_heads=28, kv_heads=4, d_head=128,
             sink=128, window=2048, streaming=2, page=64, form="bf16"),
        # continuous batching in 8 bits, small pages
        dict(name="decode_b64_ragged", kind="decode", seqs=64, low=4096, high=32768, q_heads=32, kv_heads=8, d_head=128,
             sink=64, window=2048, streaming=4, page=16, form="e4m3"),
        # the same layers in bf16, fewer requests
        dict(name="decode_b24_ragged", kind="decode", seqs=24, low=1, high=32768, q_heads=32, kv_heads=8, d_head=128,
             sink=64, window=2048, streaming=4, page=64, form="bf16"),
        # 64-wide heads in 8 bits
        dict(name="decode_d64_b8", kind="decode", seqs=8, low=12001, high=32768, q_heads=32, kv_heads=8, d_head=64,
             sink=64, window=1024, streaming=4, page=64, form="e4m3"),
        # the largest step: 16 sequences at 128K
        dict(name="decode_b16_128k", kind="decode", seqs=16, low=131072, high=131072, q_heads=32, kv_heads=8, d_head=128,
             sink=128, window=4096, streaming=4, page=128, form="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(["prompt", "prompt", "cache", "decode", "decode"])
    q_heads, kv_heads, d = rng.choice([(28, 4, 128), (32, 8, 128), (16, 2, 128), (24, 8, 128), (8, 8, 128),
                                       (40, 8, 128), (32, 8, 64), (8, 2, 64), (28, 4, 64), (16, 1, 128)])
    c = dict(kind=kind, q_heads=q_heads, kv_heads=kv_heads, d_head=d)
    if kind != "cache":
        c.update(sink=rng.choice([0, 16, 64, 128]), window=_log_int(rng, 100, 4096),
                 streaming=rng.randint(0, kv_heads))
    if kind == "prompt":
        # at most the attended work of the long listed prompt, whatever the heads
        longest = int(32768 * math.sqrt(min(1.0, 14 / q_heads)))
        high = _log_int(rng, 20, longest)
        c.update(seqs=max(1, min(100, _log_int(rng, 1, max(1, longest // high)))), high=high,
                 low=rng.randint(max(1, high // 16), high), prefix=0, fused=rng.random() < 0.5)
        if rng.random() < 0.3:
            c.update(prefix=rng.randint(1, longest), high=max(1, high // 8), low=max(1, c["low"] // 8),
                     seqs=min(4, c["seqs"]))
        return c
    c.update(page=rng.choice([16, 32, 64, 128]), form=rng.choice(["e4m3", "e4m3", "bf16"]))
    if kind == "cache":
        del c["q_heads"]
        high = _log_int(rng, 1, 32768)
        c.update(seqs=max(1, min(256, _log_int(rng, 1, max(1, 49152 // high)))), high=high,
                 low=rng.randint(max(1, high // 8), high), prefix=rng.choice([0, rng.randint(1, 20000)]))
    else:
        row = 2 * kv_heads * d * (1 if c["form"] == "e4m3" else 2)
        high = _log_int(rng, 500, 131072)
        c.update(seqs=max(1, min(128, _log_int(rng, 1, max(1, int(2.0e9 / row) // high)))), high=high,
                 low=rng.randint(1, high))
    return c


# ------------------------------------------------------------------ inputs

class State:
    pass


def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1009 + tag)


def _lens(case):
    """Tokens of each sequence, from `low` to `high`: the same in every seed, so
    that a pass of a case is always as much work."""
    r = random.Random(7919 * case["seqs"] + case["high"] + case["low"])
    return [case["high"]] + [r.randint(case["low"], case["high"]) for _ in range(case["seqs"] - 1)]


def _labels(case):
    picked = random.Random(131 * case["kv_heads"] + case["streaming"]).sample(range(case["kv_heads"]), case["streaming"])
    return [1 if h in picked else 0 for h in range(case["kv_heads"])]


def _keys(shape, seed, tag):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.bfloat16)


def _values(shape, seed, tag):
    """Rows of different sizes, as tokens' value vectors have."""
    v = torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.bfloat16)
    size = torch.randn(shape[:-1] + (1,), generator=_gen(seed, tag + 1), device="cuda").mul_(0.5).exp_()
    return v.mul_(size.to(torch.bfloat16))


def _past(case, seed, b, n):
    """K and V of sequence b's n tokens; the first is an attention sink: a large
    key and a small value."""
    k = _keys((n, case["kv_heads"], case["d_head"]), seed, 10000 + 10 * b)
    v = _values((n, case["kv_heads"], case["d_head"]), seed, 10003 + 10 * b)
    k[0] *= 8.0
    v[0] *= 0.125
    return k, v


def _power(x):
    """The row's power of two (as a float) of x [..., d]: the least one with which its
    largest finite number is at most 448."""
    f = x.float()
    m, e = torch.frexp(torch.where(torch.isfinite(f), f.abs(), 0.0).amax(-1, keepdim=True))
    return torch.where(m <= 0.875, e - 9, e - 8).clamp(E_MIN, E_MAX)


def _encode(x):
    """Codes (uint8) and powers (int8) of rows x [..., d]."""
    e = _power(x)
    codes = torch.ldexp(x.float(), -e).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), e.squeeze(-1).to(torch.int8)


def _decode(codes, powers):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), powers.unsqueeze(-1).int())


class Pool:
    """The pages' memory as the plain form sees it."""

    def __init__(self, case, pages):
        n, p, d = case["kv_heads"], case["page"], case["d_head"]
        self.form, self.page, self.pages = case["form"], p, pages
        numbers = pages * 2 * n * p * d
        if self.form == "bf16":
            self.bytes = torch.empty(2 * numbers, dtype=torch.uint8, device="cuda")
            self.data = self.bytes.view(torch.bfloat16).view(pages, 2, n, p, d)
        else:
            self.bytes = torch.empty(numbers + pages * 2 * n * p, dtype=torch.uint8, device="cuda")
            self.data = self.bytes[:numbers].view(pages, 2, n, p, d)
            self.powers = self.bytes[numbers:].view(torch.int8).view(pages, n, 2, p)
        self.bytes.fill_(255)  # what was never written may be anything: here NaN

    def write(self, k, v, page, row):
        """Rows k, v [n, kv heads, d] to `row` of `page` (both [n])."""
        for sel, x in ((0, k), (1, v)):
            if self.form == "bf16":
                self.data[page, sel, :, row] = x
            else:
                codes, powers = _encode(x)
                self.data[page, sel, :, row] = codes
                self.powers[page, :, sel, row] = powers

    def read(self, page, row):
        """The numbers at `row` of `page` (both [n]) in 32 bits: K, V [n, kv heads, d]."""
        out = []
        for sel in (0, 1):
            x = self.data[page, sel, :, row]
            out.append(x.float() if self.form == "bf16" else _decode(x, self.powers[page, :, sel, row]))
        return out


def _table(case, lens, seed):
    """Pages dealt to the sequences in a random order, some pages free: the table
    [seqs][most] with -1 past a sequence's pages, and the number of pages."""
    need = [-(-n // case["page"]) for n in lens]
    pages = sum(need) + max(2, sum(need) // 16)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed) * 31 + 5), dtype=torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table.cuda(), pages


def _places(case, table, b, first, n):
    """Page and row of positions first .. first + n - 1 of sequence b."""
    pos = torch.arange(first, first + n, device="cuda")
    return table[b, pos // case["page"]].long(), pos % case["page"]


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _sums(xs):
    out = [0]
    for x in xs:
        out.append(out[-1] + x)
    return out


def _prompt_inputs(case, seed):
    q_lens = _lens(case)
    k_lens = [n + case["prefix"] for n in q_lens]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["d_head"]
    q = _keys((sum(q_lens), hq, d), seed, 1)
    ks, vs = zip(*(_past(case, seed, b, n) for b, n in enumerate(k_lens)))
    k, v = torch.cat(ks), torch.cat(vs)
    if case["fused"] and case["prefix"] == 0:
        qkv = torch.cat([q, k, v], 1)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    return q, k, v, q_lens, k_lens


def _cache_inputs(case, seed):
    """New rows k, v of all sequences, and how many tokens each holds before and after."""
    rows = _lens(case)
    before = [case["prefix"]] * len(rows)
    ks, vs = zip(*(_past(case, seed, b, n) for b, n in enumerate(rows)))
    return torch.cat(ks), torch.cat(vs), rows, before, [a + b for a, b in zip(before, rows)]


def _decode_inputs(case, seed):
    """One query token of every sequence, and the pages that hold their keys."""
    lens = _lens(case)
    q = _keys((len(lens), case["q_heads"], case["d_head"]), seed, 1)
    table, pages = _table(case, lens, seed)
    pool = Pool(case, pages)
    for b, n in enumerate(lens):
        pool.write(*_past(case, seed, b, n), *_places(case, table, b, 0, n))
    return q, lens, table, pool


def _handle(case, pages, pool, page, form):
    from paper_2608_06849_gb300 import aoh

    return aoh.PagedCache(pages, page, case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["d_head"],
                          case.get("sink", 0), case.get("window", 1),
                          _labels(case) if "streaming" in case else [0] * case["kv_heads"],
                          form=form, max_seqs=case["seqs"], pool=pool)


def prepare(case, seed):
    s = State()
    s.case = case
    s.kind = case["kind"]
    if s.kind == "prompt":
        s.q, s.k, s.v, s.q_lens, s.k_lens = _prompt_inputs(case, seed)
        s.out = torch.empty(s.q.shape, dtype=torch.bfloat16, device="cuda")
        if own:
            # prompts need none of the pages; the handle has a pool of the least size
            s.paged = _handle(case, 1, None, 16, "bf16")
    elif s.kind == "cache":
        s.k, s.v, s.rows, s.before, after = _cache_inputs(case, seed)
        s.table, pages = _table(case, after, seed)
        s.pool = Pool(case, pages)
        s.n, s.sums = sum(s.rows), _sums(s.rows)
        s.cu, s.first, s.lens = _ints(s.sums), _ints(s.before), _ints(after)
        s.k_out, s.v_out = torch.empty_like(s.k), torch.empty_like(s.v)
        if own:
            s.paged = _handle(case, pages, s.pool.bytes, case["page"], case["form"])
    else:
        s.q, s.host_lens, s.table, s.pool = _decode_inputs(case, seed)
        s.lens = _ints(s.host_lens)
        s.out = torch.empty_like(s.q)
        if own:
            s.paged = _handle(case, s.pool.pages, s.pool.bytes, case["page"], case["form"])
    return s


# ------------------------------------------------------------------ one pass

def _attend(case, q, k, v, first):
    """Rows q [n, q heads, d] at positions first .. over keys k, v [m, kv heads, d], in 32
    bits; a row that sees no key gives zeros."""
    n, hq, d = q.shape
    m, hk, _ = k.shape
    g = hq // hk
    streaming = torch.tensor(_labels(case), device=q.device).view(hk, 1, 1, 1) == 1
    kt, vt = k.permute(1, 2, 0), v.permute(1, 0, 2)
    out = torch.empty_like(q)
    step = max(1, min(n, (1 << 29) // (hq * m)))
    for a in range(0, n, step):
        e = min(n, a + step)
        seen = max(0, min(m, first + e))
        pos = torch.arange(first + a, first + e, device=q.device).view(1, 1, -1, 1)
        j = torch.arange(seen, device=q.device).view(1, 1, 1, -1)
        hide = (j > pos) | (streaming & (j >= case["sink"]) & (pos - j >= case["window"]))
        x = q[a:e].view(e - a, hk, g, d).permute(1, 2, 0, 3).reshape(hk, g * (e - a), d)
        s = torch.matmul(x, kt[:, :, :seen]).mul_(1.0 / math.sqrt(d)).view(hk, g, e - a, seen)
        s.masked_fill_(hide, -math.inf)
        top = s.amax(-1, keepdim=True) if seen else s.new_full((hk, g, e - a, 1), -math.inf)
        s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = s.sum(-1, keepdim=True)
        o = torch.matmul(s.view(hk, g * (e - a), seen), vt[:, :seen]).view(hk, g, e - a, d)
        o = torch.where(total == 0, 0.0, o / total)
        out[a:e] = o.permute(2, 0, 1, 3).reshape(e - a, hq, d)
    return out


def run(s):
    if s.kind == "prompt":
        if own:
            s.paged.prefill(s.q, s.k, s.v, s.q_lens, s.out, k_lens=s.k_lens)
            return s.out
        qa, ka = 0, 0
        for n, m in zip(s.q_lens, s.k_lens):
            o = _attend(s.case, s.q[qa:qa + n].float(), s.k[ka:ka + m].float(), s.v[ka:ka + m].float(), m - n)
            s.out[qa:qa + n] = o.to(torch.bfloat16)
            qa, ka = qa + n, ka + m
        return s.out
    if s.kind == "cache":
        if own:
            s.paged.append(s.k, s.v, s.lens, s.table, cu_rows=s.cu)
            s.paged.read(s.table, s.cu, s.k_out, s.v_out, first=s.first)
            return s.k_out, s.v_out
        # sequence and position of every row, then all rows at once
        row = torch.arange(s.n, device="cuda")
        b = torch.searchsorted(s.cu, row, right=True) - 1
        pos = row - s.cu[b] + s.first[b]
        page, at = s.table[b, pos // s.case["page"]].long(), pos % s.case["page"]
        s.pool.write(s.k, s.v, page, at)
        for out, x in zip((s.k_out, s.v_out), s.pool.read(page, at)):
            out.copy_(x)
        return s.k_out, s.v_out
    if own:
        s.paged.decode(s.q, s.lens, s.table, s.out)
        return s.out
    for b, n in enumerate(s.host_lens):
        k, v = s.pool.read(*_places(s.case, s.table, b, 0, n))
        s.out[b:b + 1] = _attend(s.case, s.q[b:b + 1].float(), k, v, n - 1).to(torch.bfloat16)
    return s.out


# ------------------------------------------------------------------ the floor

def _pairs(case, streaming, n, m):
    """Keys seen by all of the last n rows of m positions."""
    if not streaming:
        return n * m - n * (n - 1) // 2
    s, w = case["sink"], case["window"]
    return sum(min(p + 1, s + w) for p in range(m - n, m))


def work(case):
    lens = _lens(case)
    d, hk = case["d_head"], case["kv_heads"]
    if case["kind"] == "prompt":
        labels, g = _labels(case), case["q_heads"] // hk
        m = [n + case["prefix"] for n in lens]
        pairs = sum(_pairs(case, x, a, b) for x in labels for a, b in zip(lens, m))
        return {"bytes": 2 * d * (2 * case["q_heads"] * sum(lens) + 2 * hk * sum(m)), "flops": 4 * d * g * pairs}
    row = d + 1 if case["form"] == "e4m3" else 2 * d
    if case["kind"] == "cache":
        # read and written as bf16 at the ends, written and read in the pages
        return {"bytes": sum(lens) * 2 * hk * (2 * 2 * d + 2 * row), "flops": 0}
    labels, g = _labels(case), case["q_heads"] // hk
    rows = sum(min(n, case["sink"] + case["window"]) if x else n for x in labels for n in lens)
    return {"bytes": 2 * row * rows + 2 * 2 * d * case["q_heads"] * len(lens), "flops": 4 * d * g * rows}


# ------------------------------------------------------------------ in 64 bits

def _exact_attend(case, q, k, v, first):
    """Attention by its definition: for each head the visible keys' weights, block of rows by
    block, in 64 bits."""
    n, hq, d = q.shape
    m, hk, _ = k.shape
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=q.device)
    labels = _labels(case)
    for h in range(hq):
        kv = h // (hq // hk)
        step = 1 if n == 1 else 1024
        for a in range(0, n, step):
            e = min(n, a + step)
            end = first + e
            if end <= 0:
                continue
            if labels[kv]:
                w0 = max(0, first + a - case["window"] + 1)
                keep = torch.cat([torch.arange(0, min(case["sink"], w0, end), device=q.device),
                                  torch.arange(w0, end, device=q.device)])
            else:
                keep = torch.arange(0, end, device=q.device)
            p = torch.arange(first + a, first + e, device=q.device).view(-1, 1)
            see = keep.view(1, -1) <= p
            if labels[kv]:
                see &= (keep.view(1, -1) < case["sink"]) | (p - keep.view(1, -1) < case["window"])
            s = (q[a:e, h].double() @ k[keep, kv].double().T) / math.sqrt(d)
            s = torch.where(see, s, -math.inf)
            p = torch.where(see, torch.exp(s - s.max(1, keepdim=True).values), 0.0)
            total = p.sum(1, keepdim=True)
            out[a:e, h] = torch.where(total > 0, (p @ v[keep, kv].double()) / total, 0.0)
    return out


def _exact_numbers(x):
    """What 8-bit rows hold of x [..., d]: multiples of the step at each number's size
    (3 bits behind the leading one, steps no finer than 2^-9), at most 448, times the row's
    power."""
    f = x.double()
    most = torch.where(torch.isfinite(f), f.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(most / 448.0, min=2.0 ** -200)))
    e = torch.where(most > 448.0 * torch.exp2(e), e + 1, e)       # where the logarithm was rounded
    e = torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(E_MIN, E_MAX)
    y = f / torch.exp2(e)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -30))), min=-6) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(case, seed):
    if case["kind"] == "cache":
        k, v = _cache_inputs(case, seed)[:2]
        return tuple(x.double() if case["form"] == "bf16" else _exact_numbers(x) for x in (k, v))
    if case["kind"] == "prompt":
        if work(case)["flops"] > 3.0e12:
            return None
        q, k, v, q_lens, k_lens = _prompt_inputs(case, seed)
        out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        qa, ka = 0, 0
        for n, m in zip(q_lens, k_lens):
            out[qa:qa + n] = _exact_attend(case, q[qa:qa + n], k[ka:ka + m], v[ka:ka + m], m - n)
            qa, ka = qa + n, ka + m
        return out
    lens = _lens(case)
    q = _keys((len(lens), case["q_heads"], case["d_head"]), seed, 1)
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        k, v = _past(case, seed, b, n)
        if case["form"] == "e4m3":
            k, v = _exact_numbers(k), _exact_numbers(v)
        out[b:b + 1] = _exact_attend(case, q[b:b + 1], k, v, n - 1)
    return out
