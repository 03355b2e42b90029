"""A run of the paged operators together, as a serving step uses them: page_update, append, attention over each request's new
tokens as a group and over its last token alone, rows read back; every step against the plain definitions on what the pages hold."""

import os
import sys

import numpy as np
import pytest
import torch

import shared_util
from oracle import paged as P
from paged_util import TORCH, host
from paper_2607_24331_gb300 import dck
from quant_util import values

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, BATCH, WIDTH, PAGES = 8, 2, 128, 16, 4, 30, 90


class _Layer:
    """Buffers that keep their places over all steps; `n` new tokens a step at most."""

    def __init__(self, dtype, quant, n):
        self.dtype, self.quant, kw = dtype, quant, dict(device="cuda")
        i32 = dict(dtype=torch.int32, **kw)
        if quant:
            self.caches = tuple(torch.full((PAGES, PAGE, HKV) + tail, fill, dtype=t, **kw) for tail, fill, t in
                                (((D,), 0x7f, torch.uint8), ((), float("nan"), torch.float32)) * 2)
            self.cache = dck.QuantCache.from_tensors(*self.caches, HQ, dtype)
        else:
            self.caches = tuple(torch.full((PAGES, PAGE, HKV, D), float("nan"), dtype=TORCH[dtype], **kw) for _ in range(2))
            self.cache = dck.PagedCache.from_tensors(*self.caches, HQ)
        self.rope = dck.Rope(D, 1e4)
        self.len, self.new, self.table = torch.zeros(BATCH, **i32), torch.zeros(BATCH, **i32), torch.full((BATCH, WIDTH), 1 << 30, **i32)
        self.free_pages, self.free = torch.arange(PAGES, **i32), torch.tensor([PAGES, 0], **i32)
        self.slots, self.positions, self.cu = torch.zeros(n, dtype=torch.int64, **kw), torch.zeros(n, **i32), torch.zeros(BATCH + 1, **i32)
        self.qkv = torch.zeros((n, HQ + 2 * HKV, D), dtype=TORCH[dtype], **kw)
        self.q, self.out, self.lse = (torch.zeros((n, HQ) + s, dtype=t, **kw) for s, t in
                                      (((D,), TORCH[dtype]), ((D,), TORCH[dtype]), ((), torch.float32)))
        self.last, self.last_lse = torch.zeros((BATCH, HQ, D), dtype=TORCH[dtype], **kw), torch.zeros((BATCH, HQ), **kw)
        self.back = [torch.zeros((n, HKV, D), dtype=TORCH[dtype], **kw) for _ in range(2)]
        of = (lambda q, p: q if quant else p)  # noqa: E731
        self.append, self.one = of(dck.dck_quant_append, dck.dck_paged_append), of(dck.dck_quant_decode_attention, dck.dck_paged_decode_attention)
        self.shared = of(dck.dck_quant_shared_attention, dck.dck_paged_shared_attention)
        self.bytes = of(dck.dck_quant_shared_workspace_size, dck.dck_paged_shared_workspace_size)(self.cache, n, WIDTH * PAGE, WIDTH * PAGE)
        self.bytes = max(self.bytes, of(dck.dck_quant_decode_workspace_size, dck.dck_paged_decode_workspace_size)(self.cache, BATCH, WIDTH * PAGE))
        self.ws = torch.full((self.bytes,), 255, dtype=torch.uint8, **kw)

    def step(self, owner, starts):
        n, most = owner.numel(), WIDTH * PAGE
        dck.check(dck.dck_page_update(BATCH, PAGE, PAGES, self.len, self.new, self.len, self.table, WIDTH, self.free_pages, self.free,
                                      self.free, n, self.slots, self.positions, self.cu), "dck_page_update")
        row, qkv = self.qkv.stride(0), self.qkv
        dck.check(self.append(self.cache, self.rope, qkv, row, qkv[:, HQ:], row, qkv[:, HQ + HKV:], row, n, self.positions, self.slots,
                              self.q, *self.caches), "append")
        self.rows, self.seen = self.table[owner], self.positions[:n] + 1
        group = self.len[owner[starts[:-1].long()]]
        dck.check(self.shared(self.cache, self.q, HQ * D, *self.caches, self.rows, WIDTH, self.seen, n, most, most, starts.numel() - 1,
                              starts, group, D ** -0.5, 0, 0.0, self.out, self.lse, self.ws, self.bytes), "shared attention")
        ends = (starts[1:] - 1).long()
        self.last_q = self.q[ends]
        dck.check(self.one(self.cache, self.last_q, HQ * D, *self.caches, self.rows[ends], WIDTH, self.seen[ends], ends.numel(), most,
                           D ** -0.5, 0, 0.0, self.last, self.last_lse, self.ws, self.bytes), "attention")
        if self.quant:
            dck.check(dck.dck_quant_read(self.cache, n, self.slots, *self.caches, self.back[0], HKV * D, self.back[1], HKV * D),
                      "dck_quant_read")

    def check(self, n, groups):
        assert dck.dck_last_device_error() == dck.DCK_OK
        c = dict(dtype=self.dtype, quant=self.quant)
        if self.quant:
            c.update(zip(("kcache", "k_scale", "vcache", "v_scale"), self.caches))
            k, v = values(c), values(c, "vcache", "v_scale")
            at = self.slots[:n].cpu().numpy()
            for got, want in zip(self.back, (k, v)):  # one rounding, of up to 4 bits to 8 or more: none
                assert np.array_equal(host(got[:n]), want.reshape(PAGES * PAGE, HKV, D)[at])
        else:
            k, v = (host(t) for t in self.caches)
        lens = self.seen.cpu().numpy()
        ref, rlse, weight, slack = P.paged_decode(host(self.q[:n]), k, v, self.rows.cpu().numpy(), lens, D ** -0.5)
        bo, bl = shared_util.bounds(c, D, lens.astype(np.float64), ref, rlse, weight, slack, 0.0)
        assert (np.abs(host(self.out[:n]) - ref) <= bo).all()
        assert (np.abs(host(self.lse[:n]) - rlse) <= bl).all()
        ends = np.cumsum(groups) - 1
        assert (np.abs(host(self.last[:len(ends)]) - ref[ends]) <= bo[ends]).all()
        assert (np.abs(host(self.last_lse[:len(ends)]) - rlse[ends]) <= bl[ends]).all()

    def fill(self, gen):
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=gen, device="cuda"))


def _places(counts):
    owner = torch.repeat_interleave(torch.arange(BATCH, device="cuda"), torch.tensor(counts, device="cuda"))
    groups = [c for c in counts if c]
    return owner, torch.tensor(np.cumsum([0] + groups), dtype=torch.int32, device="cuda"), groups


@pytest.mark.parametrize("way", [0, 1, 2])
@pytest.mark.parametrize("dtype,quant", [("bf16", True), ("f32", True), ("bf16", False), ("f32", False)])
def test_steps_of_a_batch(dtype, quant, way):
    """Chunks of any sizes, then steps of two tokens a request replayed from a graph, all in the same buffers."""
    before = dck.dck_set_shared_way(way)
    try:
        gen = torch.Generator(device="cuda").manual_seed(way)
        layer, held = _Layer(dtype, quant, 300), [0] * BATCH
        for counts in ([40, 7, 0, 130], [60, 1, 33, 1], [1, 1, 1, 1], [100, 90, 17, 33]):
            held = [a + b for a, b in zip(held, counts)]
            layer.fill(gen)
            layer.new.copy_(torch.tensor(held))
            owner, starts, groups = _places(counts)
            layer.step(owner, starts)
            layer.check(sum(counts), groups)
        owner, starts, groups = _places([2] * BATCH)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        layer.new.add_(2)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.step(owner, starts)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            layer.step(owner, starts)
        for _ in range(12):
            layer.new.add_(2)
            layer.fill(gen)
            graph.replay()
            torch.cuda.synchronize()
            layer.check(2 * BATCH, groups)
    finally:
        dck.dck_set_shared_way(before)


@pytest.mark.parametrize("dtype,bound", [("bf16", 0.1), ("f32", 0.1)])
def test_example_serves_from_8_bit_pages(dtype, bound):
    """Outputs against plain attention on 8-bit values: a key rounded the other way, off by 2^-3 of an element's value, moves a
    score by 2^-3 |q_e k_e| / sqrt(128), below 0.1 for elements up to 3.  Keys read back: half a step, 2^-4 of an element, of which
    a pair's turn adds two (sqrt 2 of it), and roundings of bf16."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import paged_serving
    r = paged_serving.serve(requests=9, pages=30, batch=6, dtype=dtype, check=True, longest=400, cache="8bit")
    assert r["requests"] == 9 and r["refused"] > 0 and r["worst"] <= bound and r["worst_keys"] <= 2 ** -3.5 + 2 ** -7, r
