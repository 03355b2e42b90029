"""dck_paged_decode_attention with a window or a score cap where tiles are dealt in ranges: window starts inside pages
and tiles, sequences shorter and longer than the window and empty ones, both joins, windows within a tile."""

import numpy as np
import pytest

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import decode, decode_bounds, decode_case, host

pytestmark = pytest.mark.gpu
LOOSE = 1 << 29  # a bound on the lengths that leaves only the ranges


def _check(c, hq, dtype, launches, window=0, softcap=0.0, max_len=None):
    out, lse, err = decode(c, hq, window, softcap, max_len=max_len)
    made = dck.dck_last_launch_count()
    assert err == dck.DCK_OK and made == launches, made
    d = c["q"].shape[2]
    args = [host(c[n]) for n in ("q", "kcache", "vcache")]
    ref, rlse, weight, slack = P.paged_decode(*args, c["table"].cpu().numpy(), c["lens"], float(np.float32(d ** -0.5)),
                                              window, softcap)
    n = np.minimum(c["lens"], window or max(c["lens"])).astype(np.float64)
    bo, bl = decode_bounds(dtype, d, n, ref, rlse, weight, slack, softcap)
    assert (np.abs(host(out) - ref) <= bo).all()
    assert np.array_equal(np.isneginf(host(lse)), np.isneginf(rlse))
    f = np.isfinite(rlse)
    assert (np.abs(host(lse)[f] - rlse[f]) <= bl[f]).all()


def _ragged(n, most, window, seed):
    """Lengths of 0 .. most, those at the window's edges among them, and the longest."""
    lens = np.random.default_rng(seed).integers(0, most + 1, n)
    edges = [0, 1, window - 1, window, window + 1, most]
    lens[:len(edges)] = edges
    return lens.tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,layout,n,most,window", [
    (4, 1, 64, 24, "rows", 6, 20000, 9001),      # few entries of many partials
    (8, 2, 256, 16, "joined", 10, 3000, 1205),
    (4, 2, 72, 7, "gaps", 700, 300, 101),        # many of few; rows shorter than the variant
    (8, 8, 64, 16, "heads", 1500, 200, 99),      # more sequences than lengths are kept in shared memory for
])
def test_windows_by_ranges(dtype, hq, hkv, d, page, layout, n, most, window):
    c = decode_case(hq, hkv, d, dtype, page, layout, _ragged(n, most, window, n), window=window, seed=n)
    _check(c, hq, dtype, 2, window)
    _check(c, hq, dtype, 2, window, softcap=3.0)


@pytest.mark.parametrize("dtype,window", [("bf16", 16), ("bf16", 5), ("f32", 8)])
def test_windows_within_a_tile(dtype, window):
    """No tile is shared: one launch."""
    c = decode_case(8, 8, 64, dtype, 7, "rows", _ragged(1500, 60, window, 1), window=window, seed=window)
    _check(c, 8, dtype, 1, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens", [(8, 2, 128, (3000, 1, 0, 777)), (16, 1, 64, (900, 31)), (10, 2, 80, (257, 65, 2) * 20)])
def test_caps_by_ranges(dtype, hq, hkv, d, lens):
    c = decode_case(hq, hkv, d, dtype, 16, "rows", lens, seed=d, q_std=6.0)
    for softcap in (20.0, 0.5):
        _check(c, hq, dtype, 2, softcap=softcap, max_len=LOOSE)
