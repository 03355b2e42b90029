"""Which way the calls over shared prefixes take by themselves, where the host's bounds leave no doubt."""

import pytest
import torch

from paper_2607_24331_gb300 import dck
from shared_util import attend, check, shared_case

pytestmark = pytest.mark.gpu
KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]
kinds = pytest.mark.parametrize("dtype,quant", KINDS, ids=["bf16", "f32", "q8-bf16", "q8-f32"])


def _in_way(which, f):
    before = dck.dck_set_shared_way(which)
    try:
        r = f()
        return r, dck.dck_last_launch_count()
    finally:
        dck.dck_set_shared_way(before)


@kinds
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 256), (8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("bound", [4096, 1 << 20])
def test_groups_of_single_rows_are_rows_by_themselves(dtype, quant, hq, hkv, d, bound):
    """As many groups as rows share nothing: the launches and bits of rows by themselves, whatever max_own says."""
    c = shared_case(hq, hkv, d, dtype, quant, 16, "rows", [(16 * (i % 3), [1 + 7 * i % 90]) for i in range(64)], seed=d)
    for max_own in (90, bound):
        call = lambda: attend(c, hq, max_len=bound, max_own=max_own)  # noqa: E731
        (out, lse, err), n = _in_way(0, call)
        (want, wlse, _), n_rows = _in_way(1, call)
        assert err == dck.DCK_OK and n == n_rows <= 2, (n, n_rows)
        assert torch.equal(out, want) and torch.equal(lse, wlse)
    check(c, hq, max_len=bound)


@kinds
def test_many_rows_on_a_long_prompt_share_it(dtype, quant):
    c = shared_case(8, 2, 128, dtype, quant, 16, "rows", [(320, [320 + 1 + i % 9 for i in range(64)])])
    (_, _, err), n = _in_way(0, lambda: attend(c, 8, max_len=16384, max_own=9))
    assert err == dck.DCK_OK and n == 4
    check(c, 8, max_len=16384, max_own=9)
