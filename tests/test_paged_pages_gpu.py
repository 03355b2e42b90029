"""dck_page_update against the sequential program on lists, value for value."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck

pytestmark = pytest.mark.gpu


class Pool:
    """The device state of a pool and one step on it."""

    def __init__(self, page, batch, width, n_pages, seed=0, n_free=None):
        self.page, self.n_pages, self.width = page, n_pages, width
        perm = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
        self.free_pages = torch.from_numpy(perm).cuda()
        self.free = torch.tensor([n_pages if n_free is None else n_free, 0], dtype=torch.int32, device="cuda")
        self.table = torch.full((batch, width), -9, dtype=torch.int32, device="cuda")
        self.len = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def step(self, new_len, n_tok, alias=True, stride=None):
        """Runs the call in place; returns (oracle's answer, the call's)."""
        old = self.len.cpu().numpy()
        want = P.page_update(self.page, old, new_len, self.table.cpu().numpy(), self.free_pages.cpu().numpy(),
                             int(self.free[0]), n_tok)
        B = len(new_len)
        new = torch.tensor(new_len, dtype=torch.int32, device="cuda")
        slots = torch.full((n_tok,), -77, dtype=torch.int64, device="cuda")
        positions = torch.full((n_tok,), -77, dtype=torch.int32, device="cuda")
        cu = torch.full((B + 1,), -77, dtype=torch.int32, device="cuda")
        out_len, out_free = (self.len, self.free) if alias else (torch.full_like(self.len, -77), torch.full_like(self.free, -77))
        dck.check(dck.dck_page_update(B, self.page, self.n_pages, self.len, new, out_len, self.table, self.width,
                                      self.free_pages, self.free, out_free, n_tok, slots, positions, cu), "dck_page_update")
        self.err = dck.dck_last_device_error()
        self.len, self.free = out_len, out_free
        got = dict(block_table=self.table, free_pages=self.free_pages, free=out_free, seq_len=out_len, slots=slots,
                   positions=positions, cu_new=cu)
        return want, {k: v.cpu().numpy() for k, v in got.items()}


def _same(want, got):
    for k in want:
        assert np.array_equal(want[k], got[k]), k


@pytest.mark.parametrize("page", [1, 7, 16, 256])
@pytest.mark.parametrize("batch,alias", [(1, True), (13, False), (300, True), (1025, True)])
def test_a_run_of_steps(page, batch, alias):
    rng = np.random.default_rng(page * 31 + batch)
    width = -(-400 // page)
    pool = Pool(page, batch, width, max(1, batch * width // 8), seed=batch)
    wanted = refused = 0
    for step in range(8):
        old = pool.len.cpu().numpy()
        kind = rng.integers(0, 6, batch)
        new = np.select([kind == 0, kind == 1, kind == 2, kind == 3],
                        [0, rng.integers(0, 401, batch), np.maximum(0, old - rng.integers(0, 9, batch)), old], old + 1)
        new = np.minimum(new, 400)
        n_tok = int(np.maximum(0, new - old).sum()) + int(rng.integers(0, 40))
        want, got = pool.step(new.tolist(), n_tok, alias)
        assert pool.err == dck.DCK_OK
        _same(want, got)
        refused += int(want["free"][1])
        # pages in use and free pages are distinct
        held = [p for b in range(batch) for p in got["block_table"][b, :-(-int(got["seq_len"][b]) // page)]]
        every = held + got["free_pages"][:got["free"][0]].tolist()
        assert len(set(every)) == len(every) == pool.n_pages
        wanted += n_tok
    assert wanted > 0 and (refused > 0 or batch == 1)


def test_want_of_pages_refuses_in_order():
    pool = Pool(16, 5, 8, 6)
    want, got = pool.step([32, 64, 16, 0, 1], 200)   # 2, 4, 1, 0, 1 pages: the first two fill the pool
    _same(want, got)
    assert got["seq_len"].tolist() == [32, 64, 0, 0, 0] and got["free"].tolist() == [0, 2]
    assert (got["slots"][96:112] == -1).all()
    want, got = pool.step([33, 0, 16, 0, 0], 40)     # the second ends: its pages serve the others at once
    _same(want, got)
    assert got["seq_len"].tolist() == [33, 0, 16, 0, 0] and pool.err == dck.DCK_OK


def test_a_prompt_of_many_tokens_and_the_largest_batch():
    pool = Pool(64, 3, 2000, 5000)
    _same(*pool.step([100001, 5, 20000], 130000))
    pool = Pool(16, 4096, 4, 9000)
    _same(*pool.step([1 + b % 40 for b in range(4096)], 100000))
    _same(*pool.step([(b * 7) % 64 for b in range(4096)], 200000))


def test_no_requests_and_no_tokens():
    pool = Pool(16, 0, 1, 4, n_free=3)
    want, got = pool.step([], 5)
    _same(want, got)
    pool = Pool(16, 2, 1, 4)
    _same(*pool.step([0, 0], 0))


def test_lengths_and_counts_outside_are_reported():
    def fresh():
        p = Pool(16, 3, 4, 12)
        p.step([20, 30, 40], 90)
        return p
    for new in ([21, -1, 41], [21, 65, 41]):  # a negative length, one beyond the table
        pool = fresh()
        n_tok = 2 + max(0, new[1] - 30)
        slots = torch.zeros(n_tok, dtype=torch.int64, device="cuda")
        pos = torch.zeros(n_tok, dtype=torch.int32, device="cuda")
        cu = torch.zeros(4, dtype=torch.int32, device="cuda")
        table = pool.table.clone()
        dck.check(dck.dck_page_update(3, 16, 12, pool.len, torch.tensor(new, dtype=torch.int32, device="cuda"), pool.len,
                                      pool.table, 4, pool.free_pages, pool.free, pool.free, n_tok, slots, pos, cu), "call")
        assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
        assert pool.len.tolist()[::2] == [21, 41] and pool.len.tolist()[1] == 30
        assert slots[0] >= 0 and slots[-1] >= 0 and (slots[1:-1] == -1).all()
        assert torch.equal(table[1], pool.table[1])
    # more new tokens than slots, and a free count outside the pool
    pool = fresh()
    pool.step([64, 64, 64], 100)
    assert pool.err == dck.DCK_ERR_INVALID
    pool = fresh()
    pool.free[0] = 13
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    one = torch.zeros(8, dtype=torch.int64, device="cuda")
    dck.check(dck.dck_page_update(3, 16, 12, pool.len, pool.len.clone(), pool.len, pool.table, 4, pool.free_pages,
                                  pool.free, pool.free, 1, one, one, cu), "call")
    assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
