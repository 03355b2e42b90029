"""8-bit pages and shared prefixes at the ends of what calls may be: the largest batches, more groups than the plan keeps in shared
memory, places beyond 32 bits, calls at once on two streams."""

import numpy as np
import pytest
import torch

import quant_util
from oracle import paged as P
from paged_util import TORCH, host
from paper_2607_24331_gb300 import dck
from shared_util import attend, check, shared_case
from test_quant_decode_gpu import _check

pytestmark = pytest.mark.gpu
KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]
kinds = pytest.mark.parametrize("dtype,quant", KINDS, ids=["bf16", "f32", "q8-bf16", "q8-f32"])


@pytest.fixture
def once():
    dck.dck_set_shared_way(2)
    yield
    dck.dck_set_shared_way(0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_batch(dtype):
    lens = ([1, 0, 3, 17, 2, 0, 0, 5] * 512)[:4096]
    _check(quant_util.decode_case(4, 1, 64, dtype, 4, "rows", lens, seed=1), 4)


@kinds
def test_the_largest_batch_in_groups(dtype, quant, once):
    """4096 rows: in one group, in groups of three (more than the plan keeps in shared memory), every row by itself."""
    check(shared_case(4, 2, 64, dtype, quant, 16, "rows", [(48, [49 + i % 9 for i in range(4096)])]), 4)
    check(shared_case(2, 2, 64, dtype, quant, 4, "rows", [(4 * (i % 6), [4 * (i % 6) + j for j in (1, 0, 3)]) for i in range(1365)]), 2)
    check(shared_case(2, 1, 64, dtype, quant, 4, "rows", [(8, [i % 11]) for i in range(4096)]), 2)


@kinds
def test_places_beyond_32_bits(dtype, quant, once):
    """Pages 2 MB apart (scales too), the last beyond 2^32 bytes: append, read, attention in groups and by single rows."""
    hq, hkv, d, page, n_pages = 16, 1, 128, 16, 4600
    el = 1 if quant else TORCH[dtype].itemsize
    step = (1 << 21) // el
    store = torch.uint8 if quant else TORCH[dtype]
    k, v = (torch.empty(n_pages * step, dtype=store, device="cuda").as_strided((n_pages, page, hkv, d), (step, hkv * d, d, 1)) for _ in range(2))
    caches = (k, v)
    if quant:
        ks, vs = (torch.empty(n_pages << 19, device="cuda").as_strided((n_pages, page, hkv), (1 << 19, hkv, 1)) for _ in range(2))
        caches = (k, ks, v, vs)
        cache = dck.QuantCache.from_tensors(*caches, hq, dtype)
    else:
        cache = dck.PagedCache.from_tensors(*caches, hq)
    n, rows = 200, 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn((n, hq + 2 * hkv, d), generator=gen, device="cuda").to(TORCH[dtype])
    pages = torch.tensor([4599, 4000, 2, 4598, 2049, 1025, 4301, 4302, 4303, 7, 4304, 1024, 2048], dtype=torch.int32, device="cuda")
    t = torch.arange(n, device="cuda")
    slots, positions = pages[t // page].long() * page + t % page, t.to(torch.int32)
    q = torch.zeros((n, hq, d), dtype=TORCH[dtype], device="cuda")
    append = dck.dck_quant_append if quant else dck.dck_paged_append
    row = qkv.stride(0)
    dck.check(append(cache, dck.Rope(d, 1e4), qkv, row, qkv[:, hq:], row, qkv[:, hq + hkv:], row, n, positions, slots, q, *caches), "append")
    small = {"kcache": k[pages.long()].contiguous(), "vcache": v[pages.long()].contiguous(), "dtype": dtype, "quant": quant}
    if quant:
        small["k_scale"], small["v_scale"] = ks[pages.long()].contiguous(), vs[pages.long()].contiguous()
        back = [torch.zeros((n, hkv, d), dtype=TORCH[dtype], device="cuda") for _ in range(2)]
        dck.check(dck.dck_quant_read(cache, n, slots, *caches, back[0], hkv * d, back[1], hkv * d), "read")
        for got, (c, s) in zip(back, (("kcache", "k_scale"), ("vcache", "v_scale"))):
            assert np.array_equal(host(got), quant_util.values(small, c, s).reshape(-1, hkv, d)[:n])
    # the same tokens on pages of their own, bit for bit
    i32 = dict(dtype=torch.int32, device="cuda")
    lens = list(range(n - rows + 1, n + 1))
    common = dict(q=q[n - rows:].contiguous(), lens=lens, dtype=dtype, quant=quant, seq_len=torch.tensor(lens, **i32),
                  group_start=torch.tensor([0, rows], **i32), shared_len=torch.tensor([n - rows + 1], **i32), max_own=rows)
    far = dict(common, kcache=k, vcache=v, table=pages[None].expand(rows, -1).contiguous())
    near = dict(common, table=torch.arange(len(pages), **i32)[None].expand(rows, -1).contiguous())
    near.update(small)
    if quant:
        far.update(k_scale=ks, v_scale=vs)
    for a, b in zip(attend(far, hq), attend(near, hq)):
        assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b == dck.DCK_OK
    check(near, hq)
    dck.dck_set_shared_way(1)
    for a, b in zip(attend(far, hq), attend(near, hq)):
        assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b == dck.DCK_OK


@kinds
def test_calls_at_once_on_two_streams(dtype, quant, once):
    """Each with its own workspace, in turns on both streams and from two graphs: the bits of one call alone."""
    cases = [shared_case(32, 8, 128, dtype, quant, 16, "rows", [(1600, [1600 + i for i in range(1, 40)])], seed=1),
             shared_case(32, 8, 128, dtype, quant, 16, "rows", [(960, [970, 1200, 1000]), (320, [330] * 9)], seed=2)]
    alone = [attend(c, 32)[:2] for c in cases]
    streams, work = [torch.cuda.Stream() for _ in cases], []
    for c in cases:
        caches = (c["kcache"], c["k_scale"], c["vcache"], c["v_scale"]) if quant else (c["kcache"], c["vcache"])
        cache = dck.QuantCache.from_tensors(*caches, 32, dtype) if quant else dck.PagedCache.from_tensors(*caches, 32)
        B, most = len(c["lens"]), max(c["lens"])
        size = (dck.dck_quant_shared_workspace_size if quant else dck.dck_paged_shared_workspace_size)(cache, B, most, c["max_own"])
        work.append((c, cache, caches, B, most, torch.empty(size, dtype=torch.uint8, device="cuda"), torch.zeros_like(c["q"]),
                     torch.zeros((B, 32), device="cuda")))
    call = dck.dck_quant_shared_attention if quant else dck.dck_paged_shared_attention

    def run(i):
        c, cache, caches, B, most, ws, out, lse = work[i]
        dck.check(call(cache, c["q"], 32 * 128, *caches, c["table"], c["table"].shape[1], c["seq_len"], B, most, c["max_own"],
                       c["group_start"].numel() - 1, c["group_start"], c["shared_len"], 128 ** -0.5, 0, 0.0, out, lse, ws, ws.numel()), "shared")

    def same():
        torch.cuda.synchronize()
        for (_, _, _, _, _, _, out, lse), (want, wlse) in zip(work, alone):
            assert torch.equal(out, want) and torch.equal(lse, wlse)
            out.zero_(), lse.zero_()
        torch.cuda.synchronize()
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                run(i)
    same()
    graphs = [torch.cuda.CUDAGraph() for _ in cases]
    for i, s in enumerate(streams):
        with torch.cuda.graph(graphs[i], stream=s):
            for _ in range(3):
                run(i)
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    same()
