"""The three ways of dck_paged_decode_attention (a CTA or a cluster per sequence and head, tiles dealt in ranges and joined
by a second launch) on the same inputs, queries off 16-byte boundaries, pages outside the pool in each; and the example."""

import os
import sys

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import decode, decode_bounds, decode_case, host

pytestmark = pytest.mark.gpu
LOOSE = 1 << 29  # a bound on the lengths that leaves only the ranges


def _expected(c, dtype, window=0, softcap=0.0):
    d = c["q"].shape[2]
    args = [host(c[n]) for n in ("q", "kcache", "vcache")]
    ref, rlse, weight, slack = P.paged_decode(*args, c["table"].cpu().numpy(), c["lens"], float(np.float32(d ** -0.5)),
                                              window, softcap)
    n = np.minimum(c["lens"], window or max(c["lens"])).astype(np.float64)
    return ref, rlse, *decode_bounds(dtype, d, n, ref, rlse, weight, slack, softcap)


def _near(got, want):
    out, lse, err = got
    ref, rlse, bo, bl = want
    assert err == dck.DCK_OK
    assert (np.abs(host(out) - ref) <= bo).all()
    assert np.array_equal(np.isneginf(host(lse)), np.isneginf(rlse))
    f = np.isfinite(rlse)
    assert (np.abs(host(lse)[f] - rlse[f]) <= bl[f]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,layout,lens,window,launches", [
    (32, 8, 128, 16, "rows", (777,), 0, 1),                           # clusters of eight
    (8, 2, 128, 24, "joined", (300, 0, 5, 129, 64, 1), 0, 1),         # clusters, some of their CTAs without a tile
    (16, 1, 64, 7, "rows", (900, 31), 0, 1),                          # sixteen query heads on one KV head
    (10, 2, 80, 16, "heads", (257, 65, 2), 0, 1),                     # rows shorter than the variant
    (24, 3, 72, 16, "gaps", (120, 0, 77), 50, 1),                     # the same in a window
    (8, 2, 256, 32, "rows", (100, 200), 0, 1),
    (32, 32, 128, 16, "rows", (40, 33, 1, 0, 17, 64) * 6, 0, 1),      # a CTA per sequence and four heads
    (32, 8, 64, 16, "joined", (20, 64, 3) * 20, 0, 1),
    (40, 2, 128, 16, "rows", (100, 90) * 9, 0, 1),                    # two chunks of query heads
    (8, 8, 128, 16, "rows", (3000, 50, 0, 4000, 1, 17, 900, 2500), 0, 2),
    (7, 7, 96, 16, "rows", (2000, 3100), 700, None),
])
def test_ways_agree_with_the_definition(dtype, hq, hkv, d, page, layout, lens, window, launches):
    c = decode_case(hq, hkv, d, dtype, page, layout, lens, window=window, seed=d + len(lens))
    want = _expected(c, dtype, window)
    tight = decode(c, hq, window)
    made = dck.dck_last_launch_count()
    assert launches is None or made == launches, made
    _near(tight, want)
    if not window:  # a window bounds the work by itself
        loose = decode(c, hq, max_len=LOOSE)
        assert dck.dck_last_launch_count() == 2
        _near(loose, want)
    # rows of queries off 16-byte boundaries
    B = len(lens)
    wide = torch.zeros((B, hq * d + 3), dtype=c["q"].dtype, device="cuda")
    wide[:, 1:1 + hq * d] = c["q"].reshape(B, -1)
    q = wide[:, 1:1 + hq * d].unflatten(1, (hq, d))
    for bound in (None, LOOSE):
        got = decode(c, hq, window, max_len=bound, q=q, q_stride=wide.stride(0))
        _near(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens", [(8, 2, 128, (500, 40, 600, 33)), (16, 1, 64, (500, 40, 600, 33)),
                                           (32, 32, 64, (50, 40, 60, 33) * 10), (10, 2, 80, (90, 40, 600, 33))])
@pytest.mark.parametrize("bound", [None, LOOSE])
def test_a_page_outside_the_pool_zeroes_its_sequence_alone(dtype, hq, hkv, d, lens, bound):
    c = decode_case(hq, hkv, d, dtype, 16, "rows", lens, seed=5)
    ref, rlse, err = decode(c, hq, max_len=bound)
    assert err == dck.DCK_OK
    for b, col, page in ((2, 0, -1), (2, (lens[2] - 1) // 16, 1 << 30), (0, 1, c["kcache"].shape[0])):
        keep = int(c["table"][b, col])
        c["table"][b, col] = page
        out, lse, err = decode(c, hq, max_len=bound)
        c["table"][b, col] = keep
        assert err == dck.DCK_ERR_INVALID
        assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
        rest = [i for i in range(len(lens)) if i != b]
        assert torch.equal(out[rest], ref[rest]) and torch.equal(lse[rest], rlse[rest])


def test_many_sequences_and_stale_shared_memory():
    """More sequences than lengths are kept in shared memory for, short and empty ones among them; heads shorter than the
    variant, whose rows' ends must stay zero after sums have passed through the ring."""
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 40, 1500).tolist()
    c = decode_case(4, 2, 72, "bf16", 16, "rows", lens, seed=1)
    want = _expected(c, "bf16")
    for bound in (None, LOOSE):
        _near(decode(c, 4, max_len=bound), want)
    c = decode_case(3, 3, 72, "f32", 16, "rows", lens[:300], seed=2)
    want = _expected(c, "f32")
    for bound in (None, LOOSE):
        _near(decode(c, 3, max_len=bound), want)


def test_the_largest_batch():
    lens = ([1, 0, 3, 17, 2, 0, 0, 5] * 512)[:4096]
    c = decode_case(4, 1, 64, "bf16", 4, "rows", lens, seed=1)
    want = _expected(c, "bf16")
    for bound in (None, LOOSE):
        _near(decode(c, 4, max_len=bound), want)


@pytest.mark.parametrize("dtype,bound", [("bf16", 2e-2), ("f32", 1e-5)])
def test_example_serves_requests(dtype, bound):
    """The serving example, with too few pages for all at once: every output against plain attention."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import paged_serving
    r = paged_serving.serve(requests=9, pages=30, batch=6, dtype=dtype, check=True, longest=400)
    assert r["requests"] == 9 and r["refused"] > 0 and r["worst"] <= bound, r
