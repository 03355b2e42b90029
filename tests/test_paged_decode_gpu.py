"""dck_paged_decode_attention against its plain definition in 64 bits, on caches that hold NaN wherever the call must
not look (rows past a sequence's end, other pages, rows before the window) and table entries outside the pool there."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import decode, decode_bounds, decode_case, host

pytestmark = pytest.mark.gpu


def _check(c, hq, dtype, window=0, softcap=0.0, scale=None, **kw):
    out, lse, err = decode(c, hq, window, softcap, scale, **kw)
    assert err == dck.DCK_OK
    d = c["q"].shape[2]
    scale = float(np.float32(d ** -0.5 if scale is None else scale))
    args = [host(c[n]) for n in ("q", "kcache", "vcache")]
    ref, rlse, weight, slack = P.paged_decode(*args, c["table"].cpu().numpy(), c["lens"], scale, window, softcap)
    n = np.minimum(c["lens"], window or max(c["lens"])).astype(np.float64)
    bo, bl = decode_bounds(dtype, d, n, ref, rlse, weight, slack, softcap)
    got, glse = host(out), host(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bo).all(), np.max(np.abs(got - ref) - bo)
    assert np.array_equal(np.isneginf(glse), np.isneginf(rlse))
    f = np.isfinite(rlse)
    assert (np.abs(glse[f] - rlse[f]) <= bl[f]).all(), np.max(np.abs(glse[f] - rlse[f]) - bl[f])
    return out, lse


EDGES = (0, 1, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,layout", [(16, "rows"), (1, "joined"), (24, "heads"), (100, "gaps"), (256, "joined")])
def test_lengths_at_the_edges_of_pages_and_tiles(dtype, page, layout):
    _check(decode_case(8, 2, 128, dtype, page, layout, EDGES, seed=page), 8, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(32, 32, 128), (8, 8, 64), (16, 1, 128), (10, 2, 80), (8, 2, 256), (3, 3, 8),
                                      (40, 2, 64), (9, 1, 192), (17, 1, 128), (64, 1, 64), (6, 3, 96), (7, 7, 128)])
def test_head_layouts(dtype, hq, hkv, d):
    _check(decode_case(hq, hkv, d, dtype, 16, "rows", (70, 1, 0, 513), seed=d), hq, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 16, 50, 127, 128, 1000])
def test_windows(dtype, window):
    lens = (0, 1, 49, 50, 51, 128, 129, 300, 999, 1001)
    _check(decode_case(8, 2, 64, dtype, 16, "joined", lens, window=window, seed=window), 8, dtype, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softcap_and_scales(dtype):
    c = decode_case(8, 4, 128, dtype, 32, "rows", (5, 200, 77), q_std=6.0)
    _check(c, 8, dtype, softcap=20.0)
    _check(c, 8, dtype, softcap=0.5, window=64)
    _check(c, 8, dtype, scale=0.0)
    _check(c, 8, dtype, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens", [
    (32, 8, 128, (5000,)),                        # one sequence over every SM
    (4, 1, 64, (20011, 1)),
    (8, 8, 64, (3, 9000, 0, 1, 4097, 64)),        # ragged
    (8, 2, 128, tuple([0] * 30 + [700] + [0] * 9)),
    (8, 2, 128, (33,) * 200),                     # more sequences than SMs
    (64, 8, 128, (2500, 10, 2500)),
])
def test_long_and_ragged_batches(dtype, hq, hkv, d, lens):
    _check(decode_case(hq, hkv, d, dtype, 16, "rows", lens, seed=len(lens)), hq, dtype)


def test_a_loose_bound_on_the_lengths():
    c = decode_case(8, 2, 128, "bf16", 16, "rows", (3, 600, 0, 41))
    for bound in (600, 601, 5000, 1 << 20, (1 << 31) - 1):
        _check(c, 8, "bf16", max_len=bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_needles_far_apart_in_magnitude(dtype):
    """The running maximum rises by 90 (in natural-log units) several times along the sequence, and one sequence's scores
    lie 300 below another's: sums must neither overflow nor lose the late tokens."""
    c = decode_case(4, 2, 64, dtype, 16, "rows", (3000, 3000), seed=4, q_std=1.0)
    kc, table = c["kcache"], c["table"].long()
    for i, t in enumerate((0, 17, 700, 1500, 2999)):
        for h in range(2):
            u = c["q"][0, 2 * h].float()
            kc[table[0, t // 16], t % 16, h] = (u * (90.0 * (i + 1) * 8 / (u @ u))).to(kc.dtype)
    c["q"][1] *= 20
    _check(c, 4, dtype)


def test_queries_as_views_and_without_lse():
    c = decode_case(8, 2, 128, "bf16", 16, "rows", (40, 300, 7))
    ref, rlse, _ = decode(c, 8)
    wide = torch.full((3, 12 * 128 + 2), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:1 + 8 * 128] = c["q"].reshape(3, -1)
    view = wide[:, 1:1 + 8 * 128]  # rows off 16-byte boundaries
    got, none, err = decode(c, 8, q=view.unflatten(1, (8, 128)), q_stride=wide.stride(0), lse=False)
    assert err == dck.DCK_OK and none is None and torch.equal(got, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_and_nan_entries_reach_only_their_heads(dtype):
    c = decode_case(8, 4, 64, dtype, 16, "rows", (100, 100, 1000))
    clean = decode(c, 8)[0]
    c["vcache"][c["table"][1, 2].long(), 3, 1, 5] = float("inf")
    c["vcache"][c["table"][2, 2].long(), 3, 0, 9] = float("nan")
    c["kcache"][c["table"][2, 50].long(), 3, 3, 9] = float("nan")
    got, _, err = decode(c, 8)
    assert err == dck.DCK_OK
    a, b = host(got), host(clean)
    same = np.ones_like(a, dtype=bool)
    same[1, 2:4, 5] = False
    same[2, 0:2, 9] = False
    same[2, 6:8] = False
    assert np.array_equal(a[same], b[same])
    assert np.isposinf(a[1, 2:4, 5]).all() and np.isnan(a[2, 0:2, 9]).all() and np.isnan(a[2, 6:8]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_and_pages_outside_are_reported_and_zero(dtype):
    c = decode_case(8, 2, 128, dtype, 16, "rows", (500, 40, 600, 33, 50))
    ref, rlse, _ = decode(c, 8)
    for b, change in ((0, lambda: c["seq_len"].__setitem__(0, -3)),
                      (1, lambda: c["seq_len"].__setitem__(1, 601)),
                      (2, lambda: c["table"].__setitem__((2, 20), -1)),
                      (3, lambda: c["table"].__setitem__((3, 2), c["kcache"].shape[0]))):
        keep = c["seq_len"].clone(), c["table"].clone()
        change()
        out, lse, err = decode(c, 8)
        assert err == dck.DCK_ERR_INVALID
        assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
        rest = [i for i in range(5) if i != b]
        assert torch.equal(out[rest], ref[rest]) and torch.equal(lse[rest], rlse[rest])
        c["seq_len"], c["table"] = keep
    out, lse, err = decode(c, 8)
    assert err == dck.DCK_OK and torch.equal(out, ref)
    # a table narrower than a length
    cache = dck.PagedCache.from_tensors(c["kcache"], c["vcache"], 8)
    size = dck.dck_paged_decode_workspace_size(cache, 5, 600)
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    narrow = c["table"][:, :33].contiguous()
    dck.check(dck.dck_paged_decode_attention(cache, c["q"], 1024, c["kcache"], c["vcache"], narrow, 33, c["seq_len"], 5,
                                             600, 128 ** -0.5, 0, 0.0, out, lse, ws, size), "call")
    assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
    assert (out[2] == 0).all() and torch.equal(out[[0, 1, 3, 4]], ref[[0, 1, 3, 4]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    """Pages on both sides of the 2^32nd element, keys and values in one pool."""
    d, page = 128, 16
    n_pages = (1 << 32) // (page * d) + 8
    pool = torch.empty((n_pages, page, 1, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    use = [3, n_pages - 1, n_pages - 8, 5, n_pages - 3]
    gen = torch.Generator(device="cuda").manual_seed(1)
    for p in use:
        pool[p] = torch.randn((page, 1, d), generator=gen, device="cuda").to(pool.dtype)
    small = torch.stack([pool[p] for p in use])
    q = torch.randn((1, 4, d), generator=gen, device="cuda").to(pool.dtype)
    lens = torch.tensor([75], dtype=torch.int32, device="cuda")
    big = dict(q=q, kcache=pool, vcache=pool, lens=[75], seq_len=lens,
               table=torch.tensor([use], dtype=torch.int32, device="cuda"))
    near = dict(big, kcache=small, vcache=small, table=torch.arange(5, dtype=torch.int32, device="cuda")[None])
    a, b = decode(big, 4), decode(near, 4)
    assert a[2] == b[2] == dck.DCK_OK and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    _check(near, 4, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_runs_streams_and_graphs_give_the_same_bits(dtype):
    c = decode_case(16, 4, 128, dtype, 16, "rows", (2000, 1, 0, 345, 129), seed=9)
    ref, rlse, _ = decode(c, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        assert torch.equal(decode(c, 16)[0], ref)
    with torch.cuda.stream(side):
        out, lse, err = decode(c, 16)
    torch.cuda.current_stream().wait_stream(side)
    assert err == dck.DCK_OK and torch.equal(out, ref) and torch.equal(lse, rlse)
    cache = dck.PagedCache.from_tensors(c["kcache"], c["vcache"], 16)
    size = dck.dck_paged_decode_workspace_size(cache, 5, 2000)
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dck.check(dck.dck_paged_decode_attention(cache, c["q"], 16 * 128, c["kcache"], c["vcache"], c["table"],
                                                 c["table"].stride(0), c["seq_len"], 5, 2000, 128 ** -0.5, 0, 0.0, out,
                                                 None, ws, size), "call")
    assert dck.dck_last_launch_count() >= 1
    for lens in ((2000, 1, 0, 345, 129), (3, 1, 0, 17, 100), (2000, 1, 0, 345, 129)):
        c["seq_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        want = ref if lens[0] == 2000 else decode(dict(c, lens=list(lens)), 16, max_len=2000)[0]
        assert torch.equal(out, want)


def test_parts_of_a_context_join_by_their_lse():
    c = decode_case(8, 2, 128, "f32", 16, "rows", (640,), seed=3)
    whole, lse, _ = decode(c, 8)
    parts = []
    for first, last in ((0, 16), (16, 40)):
        p = dict(c, table=c["table"][:, first:last].contiguous(), lens=[(last - first) * 16],
                 seq_len=torch.tensor([(last - first) * 16], dtype=torch.int32, device="cuda"))
        parts.append(decode(p, 8)[:2])
    w = torch.softmax(torch.stack([p[1] for p in parts]), 0)
    joined = sum(wi[..., None] * p[0] for wi, p in zip(w, parts))
    assert (joined - whole).abs().max() <= 1e-5 * whole.abs().max()
    assert (torch.logsumexp(torch.stack([p[1] for p in parts]), 0) - lse).abs().max() <= 1e-5
