"""A continuous batch on one uncompressed attention layer over a paged key-value cache.

Requests arrive with prompts, give a token per step and end; every step
  1. ``dck_page_update`` takes and returns pages and maps the step's new tokens to slots,
  2. the hidden states are projected (a library product) to queries, keys and values,
  3. ``dck_paged_append`` (``dck_quant_append`` with ``--cache 8bit``) rotates them and writes keys and values into their pages,
  4. ``dck_paged_shared_attention`` (``dck_quant_shared_attention``) attends: each new token is a row of the call with its
     request's block table and its own position + 1 as length, the rows of a prompt's chunk a group that reads
     what comes before it once.
Requests that find no page wait for the next step; where none can grow, one gives its pages back and starts anew later
(``Scheduler``).

    python examples/paged_serving.py [--requests 24] [--pages 400] [--dtype bf16|f32] [--cache full|8bit] [--check]

``--check`` recomputes every output with plain attention over each request's own keys and values (as 8 bits hold them), and
turns the cached keys of each request that ends (``dck_quant_read``) back by their positions (``dck_rope``'s transpose), to
what was projected.
"""

import argparse
import math
import os
import random
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2607_24331_gb300 import dck  # noqa: E402


class Layer:
    """One attention layer's projection, rotation, pages and per-step buffers."""

    def __init__(self, hidden, n_q, n_kv, d, page, n_pages, batch, width, max_tokens, dtype, seed=0, quant=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.n_q, self.n_kv, self.d, self.page, self.n_pages, self.batch, self.width = n_q, n_kv, d, page, n_pages, batch, width
        kw = dict(dtype=dtype, device="cuda")
        self.w = torch.randn((hidden, (n_q + 2 * n_kv) * d), generator=gen, **kw).mul_(1.5 / math.sqrt(hidden))
        self.dtype, self.quant = dtype, quant
        pool = torch.zeros((n_pages, 2, page, n_kv, d), dtype=torch.uint8 if quant else dtype, device="cuda")
        self.k, self.v = pool[:, 0], pool[:, 1]
        if quant:
            scales = torch.zeros((n_pages, 2, page, n_kv), device="cuda")
            self.caches = (self.k, scales[:, 0], self.v, scales[:, 1])
            self.cache = dck.QuantCache.from_tensors(*self.caches, n_q, "f32" if dtype == torch.float32 else "bf16")
        else:
            self.caches = (self.k, self.v)
            self.cache = dck.PagedCache.from_tensors(self.k, self.v, n_q)
        self.rope = dck.Rope(d, 1e6, scaling="linear", factor=2.0)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.len = torch.zeros(batch, **i32)
        self.table = torch.zeros((batch, width), **i32)
        self.free_pages = torch.arange(n_pages - 1, -1, -1, **i32)
        self.free = torch.tensor([n_pages, 0], **i32)
        self.slots = torch.zeros(max_tokens, dtype=torch.int64, device="cuda")
        self.positions = torch.zeros(max_tokens, **i32)
        self.cu = torch.zeros(batch + 1, **i32)
        self.max_tokens, self.max_len = max_tokens, width * page
        size = dck.dck_quant_shared_workspace_size if quant else dck.dck_paged_shared_workspace_size
        self.ws_bytes = size(self.cache, max_tokens, self.max_len, self.max_len)
        self.ws = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device="cuda")

    def step(self, new_len, owner, starts, x):
        """Grows each request to new_len (device int32 [batch]); owner [n]: the request of each new token, in the order
        of requests; starts: where each request's tokens begin (and n); x [n, hidden].  Returns (outputs [n, Hq, d],
        qkv [n, Hq + 2 Hkv, d])."""
        n = x.shape[0]
        dck.check(dck.dck_page_update(self.batch, self.page, self.n_pages, self.len, new_len, self.len, self.table,
                                      self.width, self.free_pages, self.free, self.free, n, self.slots, self.positions,
                                      self.cu), "dck_page_update")
        qkv = (x @ self.w).view(n, self.n_q + 2 * self.n_kv, self.d)
        row = qkv.stride(0)
        q = torch.empty((n, self.n_q, self.d), dtype=x.dtype, device="cuda")
        append = dck.dck_quant_append if self.quant else dck.dck_paged_append
        dck.check(append(self.cache, self.rope, qkv, row, qkv[:, self.n_q:], row, qkv[:, self.n_q + self.n_kv:], row, n,
                         self.positions, self.slots, q, *self.caches), "append")
        out = torch.empty_like(q)
        # a token that got no slot attends to nothing: its output is zero
        seen = torch.where(self.slots[:n] >= 0, self.positions[:n] + 1, 0).to(torch.int32)
        # a chunk's tokens share all of their request's up to their own; a single token shares nothing
        groups = len(starts) - 1
        begin = torch.tensor(starts, dtype=torch.int32, device="cuda")
        shared = self.len[owner[begin[:-1].long()]]
        alone = any(b - a == 1 for a, b in zip(starts, starts[1:]))
        attend = dck.dck_quant_shared_attention if self.quant else dck.dck_paged_shared_attention
        dck.check(attend(self.cache, q, self.n_q * self.d, *self.caches, self.table[owner], self.width, seen, n, self.max_len,
                         self.max_len if alone else min(n, self.max_len) or 1, groups, begin, shared, 1 / math.sqrt(self.d), 0, 0.0,
                         out, None, self.ws, self.ws_bytes), "attention")
        return out, qkv

    def keys_as_projected(self, b, n):
        """The keys of request b's first n tokens, read from its pages and turned back by their positions."""
        t = torch.arange(n, device="cuda")
        if self.quant:
            slots = self.table[b, t // self.page].long() * self.page + t % self.page
            rows, values = (torch.empty((n, self.n_kv, self.d), dtype=self.dtype, device="cuda") for _ in range(2))
            dck.check(dck.dck_quant_read(self.cache, n, slots, *self.caches, rows, self.n_kv * self.d, values, self.n_kv * self.d),
                      "dck_quant_read")
        else:
            rows = self.k[self.table[b, t // self.page].long(), t % self.page]
        dtype = dck.DCK_F32 if rows.dtype == torch.float32 else dck.DCK_BF16
        dck.check(dck.dck_rope(self.rope, rows, n, self.n_kv, self.d, dtype, self.n_kv * self.d, self.d, t.to(torch.int32), rows,
                               self.n_kv * self.d, self.d, transpose=True), "dck_rope")
        return rows


def in_8_bits(x):
    """What 8-bit pages hold of rows of finite numbers."""
    scale = 2.0 ** torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100) / 448))
    return (x / scale).float().to(torch.float8_e4m3fn).double() * scale


def plain(layer, qkv, n_before):
    """Outputs for the tokens from n_before on of one request whose qkv rows are [n, Hq + 2 Hkv, d]."""
    d, n = layer.d, qkv.shape[0]
    x = qkv.double()
    a = torch.outer(torch.arange(n, device="cuda").double(), 1e6 ** (-2.0 * torch.arange(d // 2, device="cuda").double() / d) / 2)
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    turn = lambda y: torch.cat([y[..., :d // 2] * c - y[..., d // 2:] * s, y[..., :d // 2] * s + y[..., d // 2:] * c], -1)  # noqa: E731
    rounded = lambda y: y.to(qkv.dtype).double()  # noqa: E731
    q, k = rounded(turn(x[:, :layer.n_q])), rounded(turn(x[:, layer.n_q:layer.n_q + layer.n_kv]))
    g = layer.n_q // layer.n_kv
    v = x[:, layer.n_q + layer.n_kv:]
    if layer.quant:
        k, v = in_8_bits(k), in_8_bits(v)
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    w = torch.einsum("ihd,jhd->hij", q[n_before:], k) / math.sqrt(d)
    late = torch.arange(n, device="cuda") > torch.arange(n_before, n, device="cuda")[:, None]
    return torch.einsum("hij,jhd->ihd", torch.softmax(w.masked_fill(late, -math.inf), -1), v)


class Scheduler:
    """Which requests run and how many tokens each takes, on the host; a request is (prompt tokens, answer tokens).

    While a request waits for pages none is admitted.  Where no request can grow, the last that holds pages gives them
    back: the first is never it, since with all other pages free it can grow.  So the first always ends, and so do all."""

    def __init__(self, requests, batch, chunk):
        self.waiting, self.batch, self.chunk = list(requests), batch, chunk
        self.running = [None] * batch  # [prompt left, answers left, the request]
        self.held = [0] * batch
        self.done = self.tokens = self.steps = self.refused = self.restarted = 0
        self.starved = False

    def ask(self):
        """(tokens that each slot is to hold, the slot of each new token)."""
        new, owner = [], []
        for b in range(self.batch):
            if self.running[b] is None and self.held[b] == 0 and self.waiting and not self.starved:
                request = self.waiting.pop()
                self.running[b] = [*request, request]
            r = self.running[b]
            n = 0 if r is None else min(self.chunk, r[0]) if r[0] else 1
            new.append(0 if r is None else self.held[b] + n)
            owner += [b] * n
        return new, owner

    def answer(self, new, got):
        """Takes the tokens that each slot holds now; returns the slots whose requests have ended, restarted ones among them."""
        ended, grown, self.starved = [], False, False
        for b, r in enumerate(self.running):
            n, self.held[b] = new[b] - self.held[b], got[b]
            if r is None:
                continue
            if got[b] != new[b]:
                self.starved = True
                self.refused += 1
                continue
            r[0], r[1] = (r[0] - n, r[1]) if r[0] else (0, r[1] - 1)
            self.tokens += n
            grown = True
            if r[0] == 0 and r[1] == 0:
                ended.append(b)
                self.done += 1
        if self.starved and not grown:
            last = max(b for b in range(self.batch) if self.running[b] and self.held[b])
            self.waiting.append(self.running[last][2])
            ended.append(last)
            self.restarted += 1
        for b in ended:
            self.running[b] = None
        self.steps += 1
        return ended


def serve(requests=24, pages=400, page=16, batch=8, dtype="bf16", check=False, seed=0, longest=600, n_q=8, n_kv=2, d=128,
          cache="full"):
    """Runs all requests to their ends; returns a dict of figures (if check: worst, the worst error against plain attention and,
    on pages of full width, of keys read back; worst_keys, that of keys read back alone)."""
    rng = random.Random(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    hidden, chunk = 512, 64
    width = -(-longest // page)
    work = [(rng.randint(1, longest // 2), rng.randint(1, longest // 8)) for _ in range(requests)]
    if requests and max(-(-(p + a) // page) for p, a in work) > pages:
        raise ValueError("a request needs more pages than there are: it would wait for ever")
    layer = Layer(hidden, n_q, n_kv, d, page, pages, batch, width, batch * chunk, dt, seed, cache == "8bit")
    plan = Scheduler(work, batch, chunk)
    rows = [[] for _ in range(batch)]  # each running request's qkv rows so far
    worst = worst_keys = 0.0
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    begin = time.perf_counter()
    while plan.done < requests:
        held = list(plan.held)
        new, owner = plan.ask()
        x = torch.randn((len(owner), hidden), generator=gen, device="cuda", dtype=dt)
        starts = [i for i, b in enumerate(owner) if i == 0 or owner[i - 1] != b] + [len(owner)]
        out, qkv = layer.step(torch.tensor(new, dtype=torch.int32, device="cuda"), torch.tensor(owner, dtype=torch.int64, device="cuda"),
                              starts, x)
        got = layer.len.tolist()  # the scheduler's look at what was granted
        at = 0
        for b in range(batch):
            n = max(0, new[b] - held[b])
            if n and got[b] == new[b]:
                rows[b].append(qkv[at:at + n])
                if check:
                    mine = torch.cat(rows[b])
                    want = plain(layer, mine, mine.shape[0] - n)
                    worst = max(worst, float((out[at:at + n].double() - want).abs().max() / want.abs().max()))
            elif n and check:
                assert (out[at:at + n] == 0).all()
            at += n
        for b in plan.answer(new, got):
            if check and got[b]:  # its pages are given back in the next step
                keys = torch.cat(rows[b])[:, n_q:n_q + n_kv].double()
                back = layer.keys_as_projected(b, got[b]).double()
                worst_keys = max(worst_keys, float((back - keys).abs().max() / keys.abs().max()))
                if not layer.quant:  # (8-bit pages hold keys to half a step of theirs, far more than outputs are off)
                    worst = max(worst, worst_keys)
            rows[b] = []
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    # give back the last pages
    layer.step(torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), [0, 1],
               torch.zeros((1, hidden), dtype=dt, device="cuda"))
    dck.check(dck.dck_last_device_error(), "device error")
    assert int(layer.free[0]) == pages and sorted(layer.free_pages.tolist()) == list(range(pages))
    return dict(requests=plan.done, tokens=plan.tokens, steps=plan.steps, refused=plan.refused, restarted=plan.restarted,
                seconds=took, worst=worst, worst_keys=worst_keys)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=24)
    ap.add_argument("--pages", type=int, default=400)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--cache", choices=("full", "8bit"), default="full")
    ap.add_argument("--check", action="store_true")
    o = ap.parse_args()
    r = serve(o.requests, o.pages, dtype=o.dtype, check=o.check, cache=o.cache)
    print("%(requests)d requests, %(tokens)d tokens in %(steps)d steps, %(refused)d waits for pages, %(restarted)d restarts, %(seconds).2f s" % r
          + (", worst error %.1e (keys read back: %.1e)" % (r["worst"], r["worst_keys"]) if o.check else ""))
