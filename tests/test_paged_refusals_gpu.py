"""What dck_page_update does with more new tokens than there are slots for, and with page numbers outside the pool, value
for value against the sequential program: lengths, tables, free list and slots, of the requests concerned and the others."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck

pytestmark = pytest.mark.gpu
BAD = (-1, -(1 << 31), 1 << 30)


def _step(page, n_pages, old, new, table, free_pages, n_free, n_tok):
    """(what the program on lists gives, what the call gives, its device error), on copies."""
    want = P.page_update(page, old, new, table, free_pages, n_free, n_tok, n_pages)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    B, t, length, pool, free = len(old), i32(table), i32(old), i32(free_pages), i32([n_free, 0])
    slots = torch.full((n_tok,), -77, dtype=torch.int64, device="cuda")
    positions, cu = torch.full((n_tok,), -77, dtype=torch.int32, device="cuda"), torch.full((B + 1,), -77, dtype=torch.int32, device="cuda")
    dck.check(dck.dck_page_update(B, page, n_pages, length, i32(new), length, t, t.shape[1], pool, free, free, n_tok, slots,
                                  positions, cu), "dck_page_update")
    err = dck.dck_last_device_error()
    got = dict(block_table=t, free_pages=pool, free=free, seq_len=length, slots=slots, positions=positions, cu_new=cu)
    return want, {k: v.cpu().numpy() for k, v in got.items()}, err


def _same(want, got):
    for k in want:
        assert np.array_equal(want[k], got[k]), (k, want[k], got[k])


def _state(rng, page, batch, most, spare):
    """Lengths held and wanted, tables and a free list of a pool of distinct pages."""
    old = rng.integers(0, most + 1, batch)
    kind = rng.integers(0, 6, batch)
    new = np.select([kind == 0, kind == 1, kind == 2, kind == 3],
                    [0, rng.integers(0, most + 1, batch), np.maximum(0, old - rng.integers(0, 9, batch)), old], old + 1)
    new = np.minimum(new, most)
    held = -(-old // page)
    n_pages = int(held.sum()) + spare
    perm = rng.permutation(n_pages)
    table = np.full((batch, -(-most // page)), -9)
    at = 0
    for b in range(batch):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free_pages = np.zeros(n_pages, dtype=np.int64)
    free_pages[:spare] = perm[at:]
    return n_pages, old, new, table, free_pages


def test_requests_without_slots_are_refused():
    table = [[0, -9, -9, -9], [1, 2, -9, -9], [3, -9, -9, -9], [4, -9, -9, -9]]
    # 12, 7, 1 and no new tokens in 19 slots: the third has none, although it needs no page; the fourth shrinks
    want, got, err = _step(16, 8, [16, 25, 5, 9], [28, 32, 6, 0], table, [5, 6, 7, 0, 0, 0, 0, 0], 3, 19)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [28, 32, 5, 0] and got["free"].tolist() == [3, 0]
    # 12 and 20 new tokens in 20 slots: the second takes no page, the third (a page, a token) neither
    want, got, err = _step(16, 8, [16, 25, 16, 9], [28, 45, 17, 9], table, [5, 6, 7, 0, 0, 0, 0, 0], 3, 20)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [28, 25, 16, 9] and got["free"].tolist() == [2, 0]
    assert (got["slots"][12:] == -1).all() and (got["slots"][:12] >= 0).all()
    assert np.array_equal(got["block_table"][1:], table[1:])
    # no slots at all
    want, got, err = _step(16, 8, [16, 25, 16, 9], [28, 45, 17, 2], table, [5, 6, 7, 0, 0, 0, 0, 0], 3, 0)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [16, 25, 16, 2]


def test_a_request_beyond_the_table_keeps_its_places():
    """Its tokens count (their slots are -1), so a valid one behind it may have no room: refused, not half done."""
    i32 = dict(dtype=torch.int32, device="cuda")
    length, new = torch.tensor([5, 3], **i32), torch.tensor([100, 4], **i32)
    table = torch.tensor([[0, -9], [1, -9]], **i32)
    pool, free = torch.tensor([2, 3, 0, 0], **i32), torch.tensor([2, 0], **i32)
    for n_tok, held in ((96, [5, 4]), (95, [5, 3]), (90, [5, 3])):
        seq, out = length.clone(), free.clone()
        slots, pos = torch.full((n_tok,), -77, dtype=torch.int64, device="cuda"), torch.full((n_tok,), -77, **i32)
        dck.check(dck.dck_page_update(2, 16, 4, seq, new, seq, table.clone(), 2, pool.clone(), out, out, n_tok, slots, pos,
                                      torch.zeros(3, **i32)), "dck_page_update")
        assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
        assert seq.tolist() == held and out.tolist() == [2, 0]
        assert (slots[:95] == -1).all() and (n_tok < 96 or slots[95] == 19)


@pytest.mark.parametrize("bad", BAD)
def test_a_page_outside_the_pool_in_the_list_ends_it(bad):
    table = [[0, -9, -9], [1, -9, -9], [2, -9, -9], [3, -9, -9], [4, 5, -9]]
    # two, two, one page asked for (the third request none), the last gives one back; taken from the end: 5, 9, 8, bad, 7
    want, got, err = _step(16, 12, [16, 10, 3, 16, 32], [40, 40, 4, 17, 16], table,
                           [6, 7, bad, 8, 9, 0, 0, 0, 0, 0, 0, 0], 5, 100)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [40, 10, 4, 16, 16] and got["free"].tolist() == [4, 2]
    assert got["free_pages"][:4].tolist() == [6, 7, bad, 8] and got["block_table"][1].tolist() == table[1]
    # the next step meets it again, and without it all is well
    for page, held, error in ((bad, 10, dck.DCK_ERR_INVALID), (10, 40, dck.DCK_OK)):
        want, got, err = _step(16, 12, [40, 10], [40, 40], [[0, 5, 9], [1, -9, -9]], [6, 7, page, 8] + [0] * 8, 4, 40)
        assert err == error
        _same(want, got)
        assert got["seq_len"].tolist() == [40, held]
    # a page given back counts among those of the list
    want, got, err = _step(16, 12, [16, 32], [17, 0], [[0, -9], [1, bad]], [6, 7] + [0] * 10, 2, 5)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [16, 0] and got["free"].tolist() == [4, 1]


@pytest.mark.parametrize("bad", BAD)
def test_a_page_outside_the_pool_in_a_table_refuses_its_request(bad):
    table = [[0, -9, -9], [bad, -9, -9], [2, bad, -9], [3, bad, -9]]
    # the first two grow within and beyond their page, the third beyond a full table column, the fourth stays
    want, got, err = _step(16, 8, [10, 10, 32, 20], [20, 40, 33, 20], table, [4, 5, 6, 7, 0, 0, 0, 0], 4, 60)
    assert err == dck.DCK_ERR_INVALID
    _same(want, got)
    assert got["seq_len"].tolist() == [20, 10, 33, 20] and got["free"].tolist() == [2, 0]
    assert (got["slots"][10:40] == -1).all() and got["slots"][40] >= 0
    assert np.array_equal(got["block_table"][1], table[1])


@pytest.mark.parametrize("batch", [9, 32, 33, 200, 700])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_random_steps(batch, page):
    """One CTA and a cluster; slots for all tokens or for some, bad numbers in the list, the tables, or nowhere."""
    rng = np.random.default_rng(batch * 7 + page)
    refused = errors = 0
    for turn in range(12):
        n_pages, old, new, table, free_pages = _state(rng, page, batch, 300, int(rng.integers(1, 4 * batch)))
        spare = n_pages - int((-(-old // page)).sum())
        n_new = int(np.maximum(0, new - old).sum())
        n_tok = n_new + int(rng.integers(0, 20)) if turn % 3 else int(rng.integers(0, n_new + 1))
        for _ in range(turn % 4):
            if rng.random() < 0.5:
                free_pages[rng.integers(0, spare)] = rng.choice(BAD)
            else:
                b = int(rng.integers(0, batch))
                table[b, rng.integers(0, max(1, -(-old[b] // page)))] = rng.choice(BAD)
        want, got, err = _step(page, n_pages, old, new, table, free_pages, spare, n_tok)
        _same(want, got)
        refused += int((got["seq_len"] != new).sum())
        errors += err != dck.DCK_OK
        if n_new > n_tok:
            assert err == dck.DCK_ERR_INVALID
        # a granted request's new tokens all have slots inside the pool, a refused one's none
        for b in range(batch):
            mine = got["slots"][got["cu_new"][b]:got["cu_new"][b + 1]]
            if got["seq_len"][b] == new[b] > old[b]:
                assert len(mine) == new[b] - old[b] and (mine >= 0).all() and (mine < n_pages * page).all()
            elif got["seq_len"][b] != new[b]:
                assert (mine == -1).all()
    assert refused and errors
