"""Bad rows in calls over shared prefixes, with and without a window: their lengths and their block tables, whatever these
hold, reach no other row of their groups."""

import pytest
import torch

from paper_2607_24331_gb300 import dck
from shared_util import attend, check, shared_case

pytestmark = pytest.mark.gpu
KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]
kinds = pytest.mark.parametrize("dtype,quant", KINDS, ids=["bf16", "f32", "q8-bf16", "q8-f32"])
PAGE = 16


@pytest.fixture(autouse=True, params=["once", "by rows"])
def way(request):
    dck.dck_set_shared_way(2 if request.param == "once" else 1)
    yield request.param
    dck.dck_set_shared_way(0)


def _chunk(n, rows):
    return n, [n - rows + 1 + i for i in range(rows)]


# groups, bad rows: few groups, groups of a part of a warp each, one group of many rows
SHAPES = {
    "few": ([(960, [961, 970, 965, 975]), _chunk(700, 8), (0, [40])], [1, 7, 12]),
    "many": ([(64 * (1 + i % 3), [64 * (1 + i % 3) + x for x in (6, 11, 9)]) for i in range(40)], [1, 2, 30, 118]),
    "long": ([_chunk(400, 200)], [0, 3, 100, 199]),
}


def _with_bad(c, bad, length, table):
    """The case with that length in the rows `bad`, and tables there of no pages, or ("moved") of another row's in another order."""
    d = dict(c, table=c["table"].clone(), seq_len=c["seq_len"].clone())
    for b in bad:
        d["seq_len"][b] = length
        d["table"][b] = 1 << 30
        if table == "moved":
            row = c["table"][b - 1 if b else 1]
            pages = row[row < 1 << 30]
            d["table"][b] = pages[(torch.arange(len(row), device="cuda") + 3) % len(pages)]
    return d


def _check(c, bad, window, **kw):
    good = [b for b in range(len(c["lens"])) if b not in bad]
    out, lse = check(c, 8, window=window, rows=good, expect=dck.DCK_ERR_INVALID, **kw)
    assert (out[bad] == 0).all() and torch.isneginf(lse[bad]).all()
    return out, lse


@kinds
@pytest.mark.parametrize("window", [0, 40, 64, 500])
@pytest.mark.parametrize("shape", SHAPES)
def test_bad_lengths(dtype, quant, window, shape):
    """Negative, above max_seq_len and above the table: of a window's width and more beyond every other row."""
    groups, bad = SHAPES[shape]
    c = shared_case(8, 2, 64, dtype, quant, PAGE, "rows", groups, window=window, seed=window)
    most, width = max(c["lens"]), c["table"].shape[1]
    ref = None
    for length, max_len in ((-5, most), (most + 1, most), (most + window + 1000, most), ((1 << 31) - 1, most),
                            (width * PAGE + window + 500, 1 << 20)):
        for table in ("none", "moved"):
            d = _with_bad(c, bad, length, table)
            if ref is None:
                ref = _check(d, bad, window, max_len=max_len)[0]
            else:
                out, lse, err = attend(d, 8, window=window, max_len=max_len)
                assert err == dck.DCK_ERR_INVALID and (out[bad] == 0).all() and torch.isneginf(lse[bad]).all()
                # what the good rows see is the same, and so is the arithmetic but for the split by max_len
                if max_len == most:
                    assert torch.equal(out, ref)
                else:
                    _check(d, bad, window, max_len=max_len)


@kinds
@pytest.mark.parametrize("window", [0, 64, 500])
def test_bad_lengths_and_a_shared_length_beyond_the_table(dtype, quant, window):
    """Rows that share all they see may say so by any length."""
    c = shared_case(8, 2, 64, dtype, quant, PAGE, "rows", [_chunk(510, 11)], window=window, seed=3)
    c["shared_len"].fill_(1 << 20)
    check(c, 8, window=window)
    for length, max_len in ((50000, 1000), (50000, 1 << 20), ((1 << 29) + window + 1, (1 << 31) - 1)):
        for table in ("none", "moved"):
            _check(_with_bad(c, [0, 5], length, table), [0, 5], window, max_len=max_len, max_own=20)


@kinds
@pytest.mark.parametrize("window", [0, 200])
def test_rows_of_more_own_tokens_than_said(dtype, quant, way, window):
    """Like a bad length, in calls that look at them: the longest row's table is not the group's."""
    if way == "by rows":
        pytest.skip("rows by themselves do not look at max_own")
    c = shared_case(8, 2, 64, dtype, quant, PAGE, "rows", [(320, [321, 400, 333, 325]), (0, [30, 75])], window=window, seed=5)
    for table in ("none", "moved"):
        _check(_with_bad(c, [1], 400, table), [1], window, max_own=75)


@kinds
def test_groups_of_bad_rows_alone(dtype, quant):
    c = shared_case(8, 2, 64, dtype, quant, PAGE, "rows", [(320, [321, 400, 333]), (64, [70, 71]), (0, [9])], window=64)
    bad = [3, 4, 5]
    _check(_with_bad(c, bad, 10000, "none"), bad, 64, max_len=400)


@kinds
def test_groups_of_no_rows(dtype, quant):
    """Before, between and behind others, in each of the plan's ways."""
    for groups, empty in ((SHAPES["few"][0], (0, 0, 1, 3, 3)), (SHAPES["many"][0], (0, 7, 7, 7, 40)), (SHAPES["long"][0], (0, 1, 1)),
                          ([_chunk(400, 257), _chunk(300, 130)], (0, 1, 2, 2))):
        c = shared_case(8, 2, 64, dtype, quant, PAGE, "rows", groups, seed=1)
        starts, shared = c["group_start"].tolist(), c["shared_len"].tolist()
        for at in sorted(empty, reverse=True):  # a group of no rows before group `at`
            starts.insert(at, starts[at])
            shared.insert(at, 100000)
        i32 = dict(dtype=torch.int32, device="cuda")
        d = dict(c, group_start=torch.tensor(starts, **i32), shared_len=torch.tensor(shared, **i32))
        check(d, 8)
