"""dck_paged_shared_attention and dck_quant_shared_attention against the plain definition in 64 bits, row by row, on caches
that hold NaN wherever a call must not look."""

import numpy as np
import pytest
import torch

from paper_2607_24331_gb300 import dck
from paged_util import host
from shared_util import attend, check, shared_case

pytestmark = pytest.mark.gpu
KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]


@pytest.fixture(autouse=True, params=["once", "by rows"])
def way(request):
    """Every test in both ways of the calls, whatever their rule would choose."""
    dck.dck_set_shared_way(2 if request.param == "once" else 1)
    yield request.param
    dck.dck_set_shared_way(0)


kinds = pytest.mark.parametrize("dtype,quant", KINDS, ids=["bf16", "f32", "q8-bf16", "q8-f32"])


def _chunk(n, rows):
    return n, [n - rows + 1 + i for i in range(rows)]


@kinds
@pytest.mark.parametrize("page,layout", [(16, "rows"), (1, "joined"), (24, "heads"), (100, "gaps"), (256, "joined")])
def test_prompts_and_what_follows(dtype, quant, page, layout):
    groups = [(page * 7, [page * 7 + x for x in (1, 2, 33, 300)]), (page, [page + 5, page + 9]), (0, [40, 3]), (2 * page, [65])]
    check(shared_case(8, 2, 128, dtype, quant, page, layout, groups, seed=page), 8)


@kinds
@pytest.mark.parametrize("hq,hkv,d", [(32, 32, 128), (8, 8, 64), (16, 1, 128), (10, 2, 80), (8, 2, 256), (3, 3, 8), (9, 1, 192),
                                      (6, 3, 96), (7, 7, 128), (40, 2, 64), (4, 2, 200)])
def test_head_layouts(dtype, quant, hq, hkv, d):
    groups = [(1600, [1600 + x for x in (5, 1, 44)]), (96, [96 + x for x in range(1, 12)])]
    check(shared_case(hq, hkv, d, dtype, quant, 16, "rows", groups, seed=d), hq)


@kinds
@pytest.mark.parametrize("rows", [2, 3, 16, 32, 100])
def test_chunks(dtype, quant, rows):
    groups = [_chunk(n, rows) for n in (rows, 700, 129 + rows)]
    check(shared_case(8, 2, 128, dtype, quant, 16, "rows", groups, seed=rows), 8)
    check(shared_case(4, 4, 64, dtype, quant, 24, "joined", groups, seed=rows), 4)


@kinds
def test_many_rows_and_many_groups(dtype, quant):
    check(shared_case(16, 1, 64, dtype, quant, 16, "rows", [(320, [320 + 1 + i % 50 for i in range(150)])]), 16)
    groups = [(16 * (i % 5), [16 * (i % 5) + 1 + (i * j) % 37 for j in range(1 + i % 4)]) for i in range(200)]
    check(shared_case(4, 2, 64, dtype, quant, 16, "rows", groups), 4)


@kinds
def test_long_prefixes(dtype, quant):
    groups = [(6400, [6400 + x for x in (700, 1, 64, 65)]), (20000, [20016, 20001]), (16, [17, 18, 19])]
    check(shared_case(4, 1, 128, dtype, quant, 16, "rows", groups), 4)


@kinds
def test_idle_rows_and_rows_far_behind(dtype, quant):
    """Empty rows, in groups of any kind, and rows that see little of what the others share."""
    groups = [(1600, [0, 1650, 0, 1601]), (1600, [5, 1700, 800, 1600, 1590]), (320, [0, 0, 0]), (0, [0]), (640, [0, 700]), (32, [32, 32])]
    check(shared_case(8, 2, 128, dtype, quant, 16, "rows", groups), 8)


@kinds
@pytest.mark.parametrize("window", [1, 30, 127, 500, 1000, 5000])
def test_windows(dtype, quant, window):
    groups = [(960, [960 + x for x in (1, 100, 40, 400)]), _chunk(900, 20), (480, [500, 481, 0]), (480, [490])]
    check(shared_case(8, 2, 64, dtype, quant, 16, "joined", groups, window=window, seed=window), 8, window=window)


@kinds
def test_softcap_and_scales(dtype, quant):
    c = shared_case(8, 4, 128, dtype, quant, 32, "rows", [(320, [321, 400, 333, 350, 351])], q_std=6.0)
    check(c, 8, softcap=20.0)
    check(c, 8, softcap=0.5)
    check(c, 8, scale=0.0)
    check(c, 8, scale=-0.3)


@kinds
def test_loose_bounds(dtype, quant):
    c = shared_case(8, 2, 128, dtype, quant, 16, "rows", [(320, [321, 400, 333]), _chunk(500, 9)])
    for max_len, max_own in ((500, 80), (500, 81), (5000, 500), (1 << 20, 1 << 20), ((1 << 31) - 1, (1 << 31) - 1)):
        check(c, 8, max_len=max_len, max_own=max_own)


@kinds
def test_what_a_row_may_not_see_does_not_reach_it(dtype, quant):
    """Infinities and NaN in a chunk's tokens reach the rows that see them and no others."""
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", [_chunk(300, 12), (160, [161, 170, 165])])
    clean = host(attend(c, 8)[0])
    page, off = c["table"][11, 295 // 16].long(), 295 % 16  # seen by rows of 296 tokens or more: the last five
    page2 = c["table"][12, 40 // 16].long()
    if quant:
        c["vcache"][page, off, 0, 3] = 0x7f
        c["kcache"][page, off, 1, 5] = 0x7f
        c["vcache"][page2, 40 % 16, 1, 7] = 0x7f
    else:
        c["vcache"][page, off, 0, 3] = float("inf")
        c["kcache"][page, off, 1, 5] = float("nan")
        c["vcache"][page2, 40 % 16, 1, 7] = float("nan")
    got, _, err = attend(c, 8)
    assert err == dck.DCK_OK
    got = host(got)
    same = np.ones_like(got, dtype=bool)
    same[7:12, 0:4, 3] = same[7:12, 4:8] = same[12:, 4:8, 7] = False
    assert np.array_equal(got[same], clean[same])
    assert not np.isfinite(got[~same]).any()


def test_queries_as_views_and_without_lse():
    for dtype, quant in KINDS:
        c = shared_case(8, 2, 128, dtype, quant, 16, "rows", [(320, [321, 400, 333]), (64, [70, 71])])
        ref = attend(c, 8)[0]
        wide = torch.full((5, 12 * 128 + 2), float("nan"), dtype=c["q"].dtype, device="cuda")
        wide[:, 1:1 + 8 * 128] = c["q"].reshape(5, -1)
        got, none, err = attend(c, 8, q=wide[:, 1:1 + 8 * 128].unflatten(1, (8, 128)), q_stride=wide.stride(0), lse=False)
        assert err == dck.DCK_OK and none is None and torch.equal(got, ref)


@kinds
def test_bad_rows_are_recorded_and_give_zeros(dtype, quant):
    """Lengths, own pages and own tokens beyond the bound: that row alone.  A page of the shared part: the rows that see it."""
    groups = [(6400, [6401, 6500, 6440, 6450]), (3200, [3300, 3201])]
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", groups)
    for what, rows in (("negative", [1]), ("long", [1]), ("own page", [1]), ("shared page", [0, 1, 2, 3])):
        d = dict(c, table=c["table"].clone(), seq_len=c["seq_len"].clone())
        if what == "own page":
            d["table"][1, 6450 // 16] = 1 << 20
        elif what == "shared page":
            d["table"][:4, 3] = 1 << 20
        else:
            d["seq_len"][1] = -4 if what == "negative" else 6501
        other = [b for b in range(6) if b not in rows]
        out, lse = check(d, 8, max_len=6500, rows=other, expect=dck.DCK_ERR_INVALID)
        assert (out[rows] == 0).all() and torch.isneginf(lse[rows]).all(), what


@kinds
def test_groups_that_are_none(dtype, quant, way):
    """Group starts out of order or off the batch: every output zero, and recorded.  Rows by themselves do not look at them."""
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", [(320, [321, 400, 333]), (64, [70, 71])])
    for starts in ((0, 6, 5), (1, 3, 5), (0, 3, 4), (0, -1, 5), (0, 3, 1 << 30)):
        d = dict(c, group_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        if way == "by rows":
            check(d, 8)
            continue
        out, lse, err = attend(d, 8)
        assert err == dck.DCK_ERR_INVALID and (out == 0).all() and torch.isneginf(lse).all()
    check(c, 8)


@kinds
def test_more_own_tokens_than_said(dtype, quant, way):
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", [(320, [321, 400, 333]), (0, [70, 90]), (16, [50])])
    if way == "once":
        out, lse = check(c, 8, max_own=79, rows=[0, 2, 3, 5], expect=dck.DCK_ERR_INVALID)
        assert (out[[1, 4]] == 0).all() and torch.isneginf(lse[[1, 4]]).all()
    check(c, 8, max_own=90)


@kinds
def test_a_shared_length_below_zero_is_none(dtype, quant, way):
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", [(320, [321, 400, 333]), (0, [70, 90])])
    c["shared_len"][1] = -7
    check(c, 8, expect=dck.DCK_ERR_INVALID if way == "once" else dck.DCK_OK)


def test_graphs_and_streams_give_the_same_bits():
    for dtype, quant in KINDS:
        c = shared_case(32, 8, 128, dtype, quant, 16, "rows", [(4000, [4001, 4100, 4050, 0]), _chunk(2000, 5)])
        ref, rlse, _ = attend(c, 32)
        caches = (c["kcache"], c["k_scale"], c["vcache"], c["v_scale"]) if quant else (c["kcache"], c["vcache"])
        cache = dck.QuantCache.from_tensors(*caches, 32, dtype) if quant else dck.PagedCache.from_tensors(*caches, 32)
        B = len(c["lens"])
        size = (dck.dck_quant_shared_workspace_size if quant else dck.dck_paged_shared_workspace_size)(cache, B, 4100, 100)
        ws, out, lse = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.zeros_like(c["q"]), torch.zeros((B, 32), device="cuda")

        def call():
            f = dck.dck_quant_shared_attention if quant else dck.dck_paged_shared_attention
            dck.check(f(cache, c["q"], 4096, *caches, c["table"], c["table"].shape[1], c["seq_len"], B, 4100, 100, 2,
                        c["group_start"], c["shared_len"], 128 ** -0.5, 0, 0.0, out, lse, ws, size), "shared attention")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(3):  # one behind the other, in the same workspace
                call()
            side.synchronize()
            assert torch.equal(out, ref) and torch.equal(lse, rlse)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call()
                call()
        for _ in range(3):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and torch.equal(lse, rlse)


@kinds
@pytest.mark.parametrize("window", [1, 64, 100])
def test_own_tokens_are_those_in_the_window(dtype, quant, window):
    """max_own bounds the tokens beyond the shared ones that a row sees: with a window, no more than that."""
    c = shared_case(8, 2, 64, dtype, quant, 16, "rows", [(320, [1000, 700, 333]), (0, [900])], window=window)
    check(c, 8, window=window, max_own=window)


@kinds
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (4, 4, 128), (16, 1, 64)])
def test_groups_of_many_rows(dtype, quant, hq, hkv, d):
    """Long chunks and prompts of many rows, planned in parts: odd sizes, between groups of one row, of none that sees anything
    and of rows far apart."""
    groups = [(5, [6]), _chunk(400, 257), (64, [64 + i * 7 % 50 for i in range(129)]), (0, [0, 0]), (640, [640 + i % 3 for i in range(65)]),
              (0, [9]), (320, [i * 5 % 330 for i in range(193)])]
    check(shared_case(hq, hkv, d, dtype, quant, 16, "rows", groups, seed=hq), hq)
    check(shared_case(hq, hkv, d, dtype, quant, 16, "rows", groups[:2], window=100, seed=hq), hq, window=100)
    check(shared_case(hq, hkv, d, dtype, quant, 16, "rows", [_chunk(600, 500)], seed=hq), hq)
