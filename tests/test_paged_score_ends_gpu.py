"""dck_paged_decode_attention with score caps and scales at the ends of fp32: every accepted value follows the formula."""

import numpy as np
import pytest

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import decode, decode_bounds, decode_case, host

pytestmark = pytest.mark.gpu
LARGEST = float(np.finfo(np.float32).max)
LOOSE = 1 << 29  # a bound on the lengths that leaves only the ranges


def _near(got, ref, rlse, bo, bl):
    out, lse, err = got
    assert err == dck.DCK_OK
    assert (np.abs(host(out) - ref) <= bo).all() and (np.abs(host(lse) - rlse) <= bl).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_len", [None, LOOSE])
def test_a_cap_far_above_every_score_changes_nothing(dtype, max_len):
    """c tanh(s / c) = s (1 - (s / c)^2 / 3 + ..), s itself in 64 bits for c from 1e30 on."""
    lens = (5, 200, 77)
    c = decode_case(8, 2, 128, dtype, 16, "rows", lens, seed=3)
    ref, rlse, weight, slack = P.paged_decode(*[host(c[n]) for n in ("q", "kcache", "vcache")], c["table"].cpu().numpy(),
                                              lens, float(np.float32(128 ** -0.5)))
    bo, bl = decode_bounds(dtype, 128, np.array(lens, dtype=np.float64), ref, rlse, weight, slack, 0.0)
    for softcap in (1e30, 2e30, 1e37, 1e38, 3e38, LARGEST):
        _near(decode(c, 8, softcap=softcap, max_len=max_len), ref, rlse, bo, bl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_len", [None, LOOSE])
@pytest.mark.parametrize("softcap,scale", [(1e-40, 0.1), (1e-45, -0.1), (1e-38, 3.0), (0.0, LARGEST), (0.0, -LARGEST),
                                           (30.0, LARGEST), (LARGEST, LARGEST)])
def test_queries_of_zeros_weigh_all_tokens_alike(dtype, max_len, softcap, scale):
    lens = (5, 200, 77)
    c = decode_case(8, 2, 128, dtype, 16, "rows", lens, seed=4)
    c["q"].zero_()
    ref, rlse, weight, slack = P.paged_decode(*[host(c[n]) for n in ("q", "kcache", "vcache")], c["table"].cpu().numpy(), lens, 0.0)
    bo, bl = decode_bounds(dtype, 128, np.array(lens, dtype=np.float64), ref, rlse, weight, slack, 0.0)
    _near(decode(c, 8, softcap=softcap, scale=scale, max_len=max_len), ref, rlse, bo, bl)
