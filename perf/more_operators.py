"""Rotary positions, norms and chunks over the paged cache, as measurable cases.

What a layer of a server does around its attention over pages:

  rotate   queries and keys normalised for each head (or not) and rotated by their
           positions, in one pass
  append   the same on the way into the pages: from the fused projection's q, k and v
           to rotated queries and to pages of bf16 or of 8-bit numbers with a power of
           two for each row
  attend   attention of a chunk of new tokens of every sequence over its pages

Retrieval KV heads see every earlier position, streaming heads the first `sink`
positions and the last `window`. Shapes are those of the repository's workloads
(28/4 and 32/8 heads of 128, 32/8 and 8/2 heads of 64) and generic ones.

`own` false: the operators in elementary torch operations, in 32 bits, the angles in
64. `own` true: the calls of ``paper_2608_06849_gb300.aoh``.

Rotation: of a row's first `rotated` numbers, pair i (numbers i and i + rotated / 2, or, where
`interleaved`, 2 i and 2 i + 1) turns by position * base^(-2 i / rotated), and is
multiplied by `scale`. Norm: x * w / sqrt(mean(x^2) + 1e-6), before the rotation.

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
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one token of one request, between the projection and a decode step: latency
        dict(name="rotate_step_b1", kind="rotate", seqs=1, low=1, high=1, first=4096, q_heads=28, kv_heads=4, d_head=128,
             rotated=128, base=1000000.0, interleaved=False, scale=1.0, norm="bf16", fused=False),
        # a long prompt, with norms, as slices of the fused projection's output: the largest
        dict(name="rotate_32k", kind="rotate", seqs=1, low=32768, high=32768, first=0, q_heads=32, kv_heads=8, d_head=128,
             rotated=128, base=500000.0, interleaved=False, scale=1.0, norm="fp32", fused=True),
        # a batch of chunks at far positions, small model: neighbouring pairs of half of each head, no norms
        dict(name="rotate_ragged_d64", kind="rotate", seqs=9, low=101, high=2999, first=900001, q_heads=8, kv_heads=2,
             d_head=64, rotated=32, base=10000.0, interleaved=True, scale=1.0, norm="none", fused=False),
        # one token of each of 64 sequences into 8-bit pages: latency
        dict(name="append_step_b64", kind="append", seqs=64, low=1, high=1, first=4096, q_heads=32, kv_heads=8, d_head=128,
             rotated=128, base=500000.0, interleaved=False, scale=1.0, norm="none", fused=True, page=64, form="e4m3"),
        # a scheduler's batch of prompts, normed, into 8 bits
        dict(name="append_b16_ragged", kind="append", seqs=16, low=101, high=2999, first=0, q_heads=32, kv_heads=8,
             d_head=128, rotated=128, base=1000000.0, interleaved=False, scale=1.0, norm="bf16", fused=True, page=64,
             form="e4m3"),
        # a long prompt of 64-wide heads into small bf16 pages, continuing in the middle of one
        dict(name="append_16k_d64", kind="append", seqs=1, low=16384, high=16384, first=4097, q_heads=32, kv_heads=8,
             d_head=64, rotated=64, base=10000.0, interleaved=False, scale=1.1386, norm="none", fused=True, page=16,
             form="bf16"),
        # five drafted tokens of one chat verified: latency
        dict(name="attend_verify_b1", kind="attend", seqs=1, low=5, high=5, past_low=4096, past_high=4096, q_heads=28,
             kv_heads=4, d_head=128, sink=128, window=2048, streaming=2, page=64, form="bf16", fused=False),
        # drafted tokens of 32 requests over small 8-bit pages
        dict(name="attend_verify_b32", kind="attend", seqs=32, low=2, high=5, past_low=1000, past_high=16000, q_heads=32,
             kv_heads=8, d_head=128, sink=64, window=2048, streaming=4, page=16, form="e4m3", fused=True),
        # a chunk of a long prompt, bf16 pages
        dict(name="attend_chunk_2k", kind="attend", seqs=1, low=2048, high=2048, past_low=30001, past_high=30001,
             q_heads=28, kv_heads=4, d_head=128, sink=128, window=2048, streaming=2, page=64, form="bf16", fused=True),
        # a chunk of an 8-bit cache: the largest
        dict(name="attend_chunk_8k", kind="attend", seqs=1, low=8192, high=8192, past_low=16384, past_high=16384,
             q_heads=32, kv_heads=8, d_head=128, sink=64, window=2048, streaming=0, page=128, form="e4m3", fused=False),
        # a step that mixes chunks of four prompts, 8-bit pages, half of the heads streaming
        dict(name="attend_b4_ragged", kind="attend", seqs=4, low=301, high=1500, past_low=1, past_high=8001, q_heads=32,
             kv_heads=8, d_head=128, sink=64, window=512, streaming=4, page=64, form="e4m3", fused=True),
        # a mixed batch of 64-wide heads: single tokens, drafts and short chunks
        dict(name="attend_mixed_d64", kind="attend", seqs=24, low=1, high=200, past_low=0, past_high=6000, q_heads=32,
             kv_heads=8, d_head=64, sink=16, window=1000, streaming=4, page=32, form="bf16", fused=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(["rotate", "append", "attend", "attend"])
    q_heads, kv_heads, d = rng.choice([(28, 4, 128), (32, 8, 128), (16, 2, 128), (24, 8, 128), (8, 8, 128),
                                       (40, 8, 128), (32, 8, 64), (8, 2, 64), (28, 4, 64), (16, 1, 128)])
    c = dict(kind=kind, q_heads=q_heads, kv_heads=kv_heads, d_head=d, fused=rng.random() < 0.5)
    if kind != "rotate":
        c.update(page=rng.choice([16, 32, 64, 128]), form=rng.choice(["e4m3", "e4m3", "bf16"]))
    if kind != "attend":
        most = int(32768 * 40 * 128 / ((q_heads + 2 * kv_heads) * d) / (1 if kind == "rotate" else 2))
        high = _log_int(rng, 1, min(most, 32768))
        c.update(seqs=max(1, min(256, _log_int(rng, 1, max(1, most // high)))), high=high,
                 low=rng.randint(max(1, high // 8), high),
                 first=rng.choice([0, rng.randint(1, 20000), rng.randint(1, 1000000 if kind == "rotate" else 60000)]),
                 rotated=rng.choice([d, d, d // 2, d // 4]), base=rng.choice([10000.0, 500000.0, 1000000.0]),
                 interleaved=rng.random() < 0.3, scale=rng.choice([1.0, 1.0, 1.1386]),
                 norm=rng.choice(["none", "bf16", "fp32"]))
        if kind == "append":
            c["seqs"] = max(1, min(c["seqs"], 500000 // (c["first"] + high)))
        return c
    c.update(sink=rng.choice([0, 16, 64, 128]), window=_log_int(rng, 100, 4096), streaming=rng.randint(0, kv_heads))
    # at most the scores of the largest listed chunk, whatever the heads, and as much cache as 16 x 32K
    most = 8192 * 24576 * 32 // q_heads
    high = _log_int(rng, 1, 8192)
    past = _log_int(rng, 16, min(65536, max(64, most // high - high)))
    seqs = min(most // (high * (past + high)), 524288 // (past + high))
    c.update(seqs=max(1, min(128, _log_int(rng, 1, max(1, seqs)))), high=high, low=rng.randint(max(1, high // 8), high),
             past_high=past, past_low=rng.randint(0, past))
    return c


# ------------------------------------------------------------------ inputs

class State:
    pass


def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1009 + tag)


def _spread(case, low, high, tag):
    """A number from `low` to `high` for each sequence, the first one `high`: the same in every
    seed, so that a pass of a case is always as much work."""
    r = random.Random(7919 * case["seqs"] + high + low + tag)
    return [high] + [r.randint(low, high) for _ in range(case["seqs"] - 1)]


def _rows_of(case):
    return _spread(case, case["low"], case["high"], 0)


def _pasts(case):
    """Tokens that the cache holds of each sequence before the call."""
    if case["kind"] == "attend":
        return _spread(case, case["past_low"], case["past_high"], 1)
    return [case["first"]] * case["seqs"]


def _labels(case):
    picked = random.Random(131 * case["kv_heads"] + case["streaming"]).sample(range(case["kv_heads"]), case["streaming"])
    return [1 if h in picked else 0 for h in range(case["kv_heads"])]


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _sums(xs):
    out = [0]
    for x in xs:
        out.append(out[-1] + x)
    return out


def _normal(shape, seed, tag):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.bfloat16)


def _values(shape, seed, tag):
    """Rows of different sizes, as tokens' value vectors have."""
    v = torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.bfloat16)
    size = torch.randn(shape[:-1] + (1,), generator=_gen(seed, tag + 1), device="cuda").mul_(0.5).exp_()
    return v.mul_(size.to(torch.bfloat16))


def _projected(case, seed, n):
    """q, k, v of n rows; where `fused`, slices of one tensor."""
    hq, hk, d = case["q_heads"], case["kv_heads"], case["d_head"]
    q, k, v = _values((n, hq, d), seed, 1), _values((n, hk, d), seed, 3), _values((n, hk, d), seed, 5)
    if case["fused"]:
        qkv = torch.cat([q, k, v], 1)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    return q, k, v


def _norms(case, seed):
    """Norm weights of queries and keys, near one, or None."""
    if case["norm"] == "none":
        return None, None
    t = torch.bfloat16 if case["norm"] == "bf16" else torch.float32
    return [(1.0 + 0.2 * torch.randn(case["d_head"], generator=_gen(seed, tag), device="cuda")).to(t) for tag in (7, 8)]


def _frequencies(case):
    return [case["base"] ** (-2.0 * i / case["rotated"]) for i in range(case["rotated"] // 2)]


def _positions(case):
    """Positions of all rows, sequence behind sequence; in a rotation alone each starts elsewhere."""
    step = 7777 if case["kind"] == "rotate" else 0
    return torch.cat([torch.arange(f + step * b, f + step * b + n, dtype=torch.int32, device="cuda")
                      for b, (f, n) in enumerate(zip(_pasts(case), _rows_of(case)))])


class Pool:
    """The pages' memory as the plain form sees it."""

    def __init__(self, case, pages):
        n, p, d = case["kv_heads"], case["page"], case["d_head"]
        self.form, self.page, self.pages = case["form"], p, pages
        numbers = pages * 2 * n * p * d
        if self.form == "bf16":
            self.bytes = torch.zeros(2 * numbers, dtype=torch.uint8, device="cuda")
            self.data = self.bytes.view(torch.bfloat16).view(pages, 2, n, p, d)
        else:
            self.bytes = torch.zeros(numbers + pages * 2 * n * p, dtype=torch.uint8, device="cuda")
            self.data = self.bytes[:numbers].view(pages, 2, n, p, d)
            self.powers = self.bytes[numbers:].view(torch.int8).view(pages, n, 2, p)

    def write(self, k, v, page, row):
        """Rows k, v [n, kv heads, d], in 32 bits or bf16, to `row` of `page` (both [n])."""
        for sel, x in ((0, k), (1, v)):
            if self.form == "bf16":
                self.data[page, sel, :, row] = x.to(torch.bfloat16)
                continue
            f = x.float()
            m, e = torch.frexp(torch.where(torch.isfinite(f), f.abs(), 0.0).amax(-1, keepdim=True))
            e = torch.where(m <= 0.875, e - 9, e - 8).clamp(E_MIN, E_MAX)
            self.data[page, sel, :, row] = torch.ldexp(f, -e).to(torch.float8_e4m3fn).view(torch.uint8)
            self.powers[page, :, sel, row] = e.squeeze(-1).to(torch.int8)

    def read(self, page, row, sel):
        """K (sel 0) or V (1) at `row` of `page` in 32 bits: [..., kv heads, d]."""
        x = self.data[page, sel, :, row]
        if self.form == "bf16":
            return x.float()
        return torch.ldexp(x.view(torch.float8_e4m3fn).float(), self.powers[page, :, sel, row].unsqueeze(-1).int())


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


def _cached(case, seed, b, n):
    """K and V of sequence b's n cached tokens; the first is an attention sink: a large
    key and a small value."""
    k = _normal((n, case["kv_heads"], case["d_head"]), seed, 10000 + 10 * b)
    v = _values((n, case["kv_heads"], case["d_head"]), seed, 10003 + 10 * b)
    k[0] *= 8.0
    v[0] *= 0.125
    return k, v


def _queries(case, seed, n):
    hq, hk, d = case["q_heads"], case["kv_heads"], case["d_head"]
    q = _normal((n, hq, d), seed, 1)
    if case["fused"]:
        q = torch.cat([q, _normal((n, 2 * hk, d), seed, 2)], 1)[:, :hq]
    return q


def prepare(case, seed):
    s = State()
    s.case, s.kind = case, case["kind"]
    rows = _rows_of(case)
    after = [a + b for a, b in zip(_pasts(case), rows)]
    n = sum(rows)
    if s.kind == "attend":
        s.q_lens, s.k_lens = rows, after
        s.q = _queries(case, seed, n)
        s.out = torch.empty((n, case["q_heads"], case["d_head"]), dtype=torch.bfloat16, device="cuda")
        s.table, pages = _table(case, after, seed)
        s.lens, s.cu = _ints(after), _ints(_sums(rows))
        s.pool = Pool(case, pages)
        for b, m in enumerate(after):
            pos = torch.arange(m, device="cuda")
            s.pool.write(*_cached(case, seed, b, m), s.table[b, pos // case["page"]].long(), pos % case["page"])
    else:
        s.q, s.k, s.v = _projected(case, seed, n)
        s.q_norm, s.k_norm = _norms(case, seed)
        s.q_out = torch.empty(s.q.shape, dtype=torch.bfloat16, device="cuda")
        s.k_out, s.v_out = (torch.empty(s.k.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s.positions = _positions(case)
        s.frequencies = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        if s.kind == "append":
            s.table, pages = _table(case, after, seed)
            s.lens, s.cu, s.first = _ints(after), _ints(_sums(rows)), _ints(_pasts(case))
            s.pool = Pool(case, pages)
    if own:
        from paper_2608_06849_gb300 import aoh

        if s.kind != "attend":
            s.rope = aoh.Rope(inv_freq=_frequencies(case), interleaved=case["interleaved"], scale=case["scale"])
        if s.kind != "rotate":
            s.paged = aoh.PagedCache(pages, case["page"], case["q_heads"], case["kv_heads"], case["d_head"],
                                     case.get("sink", 0), case.get("window", 1),
                                     _labels(case) if "streaming" in case else [0] * case["kv_heads"],
                                     form=case["form"], max_seqs=case["seqs"], pool=s.pool.bytes)
    return s


# ------------------------------------------------------------------ one pass

def _rotate(s, x, w, positions):
    """Rows x [n, heads, d] normed by w (or not) and rotated, in 32 bits."""
    c = s.case
    x, r = x.float(), c["rotated"]
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    angle = positions.double().unsqueeze(-1) * s.frequencies
    cos, sin = ((f(angle) * c["scale"]).float().unsqueeze(1) for f in (torch.cos, torch.sin))
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _attend(s):
    """All sequences at once, padded to the longest: their rows, and their keys, out of the pages."""
    c = s.case
    hq, hk, d = c["q_heads"], c["kv_heads"], c["d_head"]
    B, n, m, g = c["seqs"], max(s.q_lens), max(s.k_lens), hq // hk
    i, j = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    rows = s.cu[1:] - s.cu[:-1]
    there = i < rows.view(B, 1)
    at = torch.where(there, s.cu[:-1].view(B, 1) + i, 0)
    q = s.q[at].float().view(B, n, hk, g, d).permute(0, 2, 3, 1, 4).reshape(B, hk, g * n, d)
    held = j < s.lens.view(B, 1)
    page = torch.where(held, s.table[:, j // c["page"]], 0).long()
    x = torch.where(held.view(B, m, 1, 1), s.pool.read(page, (j % c["page"]).expand(B, m), 0), 0.0)
    scores = torch.matmul(q, x.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(d)).view(B, hk, g, n, m)
    pos = (s.lens - rows).view(B, 1, 1, 1, 1) + i.view(n, 1)
    streaming = torch.tensor(_labels(c), device="cuda").view(hk, 1, 1, 1) == 1
    scores.masked_fill_((j > pos) | (streaming & (j >= c["sink"]) & (pos - j >= c["window"])), -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    x = torch.where(held.view(B, m, 1, 1), s.pool.read(page, (j % c["page"]).expand(B, m), 1), 0.0)
    o = torch.matmul(scores.view(B, hk, g * n, m), x.permute(0, 2, 1, 3)).view(B, hk, g, n, d)
    o = torch.where(total == 0, 0.0, o / total).permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)
    s.out[at[there]] = o[there].to(torch.bfloat16)


def run(s):
    c = s.case
    if s.kind == "rotate":
        if own:
            from paper_2608_06849_gb300 import aoh

            aoh.aoh_norm_rotate(s.rope, s.q, s.k, s.positions, s.q_out, s.k_out, q_norm=s.q_norm, k_norm=s.k_norm, eps=EPS)
        else:
            s.q_out.copy_(_rotate(s, s.q, s.q_norm, s.positions))
            s.k_out.copy_(_rotate(s, s.k, s.k_norm, s.positions))
        return s.q_out, s.k_out
    if s.kind == "attend":
        if own:
            s.paged.attend(s.q, s.q_lens, s.lens, s.table, s.out, k_lens=s.k_lens)
        else:
            _attend(s)
        return s.out
    # pages of bf16 are an output as they are, 8-bit ones are read back as what they stand for
    if own:
        s.paged.append_rotated(s.rope, s.q, s.k, s.v, s.lens, s.table, s.q_out, cu_rows=s.cu, q_norm=s.q_norm,
                               k_norm=s.k_norm, eps=EPS)
        if c["form"] == "bf16":
            return s.q_out, s.pool.data
        s.paged.read(s.table, s.cu, s.k_out, s.v_out, first=s.first)
        return s.q_out, s.k_out, s.v_out
    row = torch.arange(s.q.shape[0], device="cuda")
    b = torch.searchsorted(s.cu, row, right=True) - 1
    pos = row - s.cu[b] + s.first[b]
    page, at = s.table[b, pos // c["page"]].long(), pos % c["page"]
    s.q_out.copy_(_rotate(s, s.q, s.q_norm, pos))
    s.pool.write(_rotate(s, s.k, s.k_norm, pos), s.v, page, at)
    if c["form"] == "bf16":
        return s.q_out, s.pool.data
    s.k_out.copy_(s.pool.read(page, at, 0))
    s.v_out.copy_(s.pool.read(page, at, 1))
    return s.q_out, s.k_out, s.v_out


# ------------------------------------------------------------------ the floor

def _pairs(case, streaming, n, m):
    """Keys seen by all of the last n rows of m positions."""
    if not streaming:
        return n * m - n * (n - 1) // 2
    s, w = case["sink"], case["window"]
    return sum(min(p + 1, s + w) for p in range(m - n, m))


def _seen(case, streaming, n, m):
    """Keys that one at least of the last n rows of m positions sees."""
    if not streaming:
        return m
    first = max(0, m - n - case["window"] + 1)  # of the first row's window
    return m - first + min(case["sink"], first)


def work(case):
    rows, d, hq, hk = _rows_of(case), case["d_head"], case["q_heads"], case["kv_heads"]
    n = sum(rows)
    if case["kind"] == "rotate":
        return {"bytes": 4 * d * (hq + hk) * n, "flops": 0}
    row = d + 1 if case["form"] == "e4m3" else 2 * d
    if case["kind"] == "append":
        # 8-bit pages are read back too
        return {"bytes": n * (4 * d * hq + 2 * hk * (2 * d + row + (2 * d + row if case["form"] == "e4m3" else 0))),
                "flops": 0}
    after = [a + b for a, b in zip(_pasts(case), rows)]
    labels, g = _labels(case), hq // hk
    pairs = sum(_pairs(case, x, a, b) for x in labels for a, b in zip(rows, after))
    seen = sum(_seen(case, x, a, b) for x in labels for a, b in zip(rows, after))
    return {"bytes": 4 * d * hq * n + 2 * row * seen, "flops": 4 * d * g * pairs}


# ------------------------------------------------------------------ in 64 bits

def _exact_numbers(x):
    """What 8-bit rows hold of x [..., d]: multiples of the step at each number's size
    (3 bits behind the leading one, steps no finer than 2^-9), at most 448, times the row's
    power."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(most / 448.0, min=2.0 ** -200)))
    e = torch.where(most > 448.0 * torch.exp2(e), e + 1, e)       # where the logarithm was rounded
    e = torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(E_MIN, E_MAX)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -30))), min=-6) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def _exact_rotated(case, x, w, positions):
    """Each pair of numbers as a complex number, times one on the circle."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    r = case["rotated"]
    head, rest = x[..., :r], x[..., r:]
    pairs = head.unflatten(-1, (r // 2, 2)) if case["interleaved"] else head.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    f = torch.tensor(_frequencies(case), dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.full_like(f, case["scale"]).expand(len(positions), -1), positions.double()[:, None] * f[None])
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
    z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, rest], -1)


def _exact_attend(case, q, k, v, first):
    """Attention by its definition: for each head the visible keys' weights, block of rows by
    block."""
    n, hq, d = q.shape
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=q.device)
    labels = _labels(case)
    for h in range(hq):
        kv = h // (hq // k.shape[1])
        for a in range(0, n, 1024):
            e = min(n, a + 1024)
            end = first + e
            keep = torch.arange(0, end, device=q.device)
            if labels[kv]:
                w0 = max(0, first + a - case["window"] + 1)
                keep = keep[(keep < case["sink"]) | (keep >= w0)]
            p = torch.arange(first + a, end, device=q.device).view(-1, 1)
            see = keep.view(1, -1) <= p
            if labels[kv]:
                see &= (keep.view(1, -1) < case["sink"]) | (p - keep.view(1, -1) < case["window"])
            x = (q[a:e, h].double() @ k[keep, kv].double().T) / math.sqrt(d)
            x = torch.softmax(torch.where(see, x, -math.inf), -1)
            out[a:e, h] = x @ v[keep, kv].double()
    return out


def exact(case, seed):
    rows = _rows_of(case)
    n = sum(rows)
    if case["kind"] == "attend":
        if work(case)["flops"] > 3.0e12:
            return None
        q = _queries(case, seed, n)
        out = torch.empty((n, case["q_heads"], case["d_head"]), dtype=torch.float64, device="cuda")
        at = 0
        for b, (a, m) in enumerate(zip(rows, _pasts(case))):
            k, v = (x.double() for x in _cached(case, seed, b, m + a))
            if case["form"] == "e4m3":
                k, v = _exact_numbers(k), _exact_numbers(v)
            out[at:at + a] = _exact_attend(case, q[at:at + a], k, v, m)
            at += a
        return out
    q, k, v = _projected(case, seed, n)
    wq, wk = _norms(case, seed)
    p = _positions(case)
    q, k = _exact_rotated(case, q, wq, p), _exact_rotated(case, k, wk, p)
    if case["kind"] == "rotate":
        return q, k
    if case["form"] == "e4m3":
        return q, _exact_numbers(k), _exact_numbers(v.double())
    after = [a + b for a, b in zip(_pasts(case), rows)]
    table, pages = _table(case, after, seed)
    pool = torch.zeros((pages, 2, case["kv_heads"], case["page"], case["d_head"]), dtype=torch.float64, device="cuda")
    b = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), _ints(rows).long())
    page, row = table[b, p.long() // case["page"]].long(), p.long() % case["page"]
    pool[page, 0, :, row] = k
    pool[page, 1, :, row] = v.double()
    return q, pool
