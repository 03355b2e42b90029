"""dck_quant_append writes the rows of its slots and nothing else: codes and scales of both caches, with all that lies between
and behind their rows, looked at each for itself."""

import numpy as np
import pytest
import torch

from paper_2607_24331_gb300 import dck
from paged_util import ROPES, TORCH
from quant_util import code_pair

pytestmark = pytest.mark.gpu
FILL = 0x55


def _whole(view):
    while view._base is not None:
        view = view._base
    return view


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("rows", 16), ("joined", 24), ("heads", 1), ("gaps", 100), ("gaps", 3)])
@pytest.mark.parametrize("setting", [ROPES[0], ROPES[5], {}], ids=["half", "six", "none"])
@pytest.mark.parametrize("hkv,d,n", [(2, 128, 1), (3, 72, 45), (1, 200, 300), (5, 64, 40), (2, 256, 9)])
def test_nothing_else_is_written(dtype, layout, page, setting, hkv, d, n):
    rng = np.random.default_rng(n + d)
    n_pages = -(-n // page) + 2
    kw = dict(setting)
    rope = dck.Rope(kw.pop("rotary_dim"), kw.pop("theta"), **kw) if kw else None
    kv = torch.from_numpy(rng.standard_normal((n, 2 * hkv, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    if n > 1:
        slots[::7] = -1
    kc, ks, vc, vs = code_pair(layout, n_pages, page, hkv, d, fill=FILL)
    cache = dck.QuantCache.from_tensors(kc, ks, vc, vs, hkv, dtype)
    pos = torch.from_numpy(rng.integers(0, 100000, n).astype(np.int32)).cuda()
    row = kv.stride(0)
    dck.check(dck.dck_quant_append(cache, rope, None, 0, kv, row, kv[:, hkv:], row, n, pos, torch.from_numpy(slots).cuda(), None,
                                   kc, ks, vc, vs), "dck_quant_append")
    assert dck.dck_last_device_error() == dck.DCK_OK
    keep = slots[slots >= 0]
    p, o = (torch.from_numpy(x).cuda() for x in (keep // page, keep % page))
    for c, s in ((kc, ks), (vc, vs)):  # what was to be written has been
        assert not torch.isnan(s[p, o]).any() and (c[p, o] != FILL).any(-1).all()
        c[p, o], s[p, o] = FILL, float("nan")
    for c in (kc, vc):  # (a joined buffer twice)
        assert _whole(c).numel() >= c.numel() and (_whole(c) == FILL).all()
    for s in (ks, vs):
        assert _whole(s).numel() >= s.numel() and torch.isnan(_whole(s)).all()
