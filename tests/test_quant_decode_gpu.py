"""dck_quant_decode_attention against its plain definition in 64 bits, on caches whose codes and scales are NaN wherever the
call must not look and whose table entries lie outside the pool there."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import host
from quant_util import decode, decode_bounds, decode_case, values

pytestmark = pytest.mark.gpu


def _check(c, hq, window=0, softcap=0.0, scale=None, **kw):
    out, lse, err = decode(c, hq, window, softcap, scale, **kw)
    assert err == dck.DCK_OK
    d, hkv = c["q"].shape[2], c["kcache"].shape[2]
    scale = float(np.float32(d ** -0.5 if scale is None else scale))
    args = [host(c["q"]), values(c), values(c, "vcache", "v_scale")]
    ref, rlse, weight, slack = P.paged_decode(*args, c["table"].cpu().numpy(), c["lens"], scale, window, softcap)
    n = np.minimum(c["lens"], window or max(c["lens"])).astype(np.float64)
    most = float(np.nan_to_num(c["v_scale"].cpu().numpy().astype(np.float64), nan=0.0).max())
    bo, bl = decode_bounds(c["dtype"], hq // hkv, d, n, ref, rlse, weight, slack, softcap, most)
    got, glse = host(out), host(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bo).all(), np.max(np.abs(got - ref) - bo)
    assert np.array_equal(np.isneginf(glse), np.isneginf(rlse))
    f = np.isfinite(rlse)
    assert (np.abs(glse[f] - rlse[f]) <= bl[f]).all(), np.max(np.abs(glse[f] - rlse[f]) - bl[f])
    return out, lse


EDGES = (0, 1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,layout", [(16, "rows"), (1, "joined"), (24, "heads"), (100, "gaps"), (256, "joined")])
def test_lengths_at_the_edges_of_pages_and_tiles(dtype, page, layout):
    _check(decode_case(8, 2, 128, dtype, page, layout, EDGES, seed=page), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(32, 32, 128), (8, 8, 64), (16, 1, 128), (10, 2, 80), (8, 2, 256), (3, 3, 8), (40, 2, 64),
                                      (9, 1, 192), (17, 1, 128), (64, 1, 64), (6, 3, 96), (7, 7, 128), (12, 1, 56), (4, 2, 200)])
def test_head_layouts(dtype, hq, hkv, d):
    _check(decode_case(hq, hkv, d, dtype, 16, "rows", (70, 1, 0, 513), seed=d), hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 16, 50, 127, 128, 1000])
def test_windows(dtype, window):
    lens = (0, 1, 49, 50, 51, 128, 129, 300, 999, 1001)
    _check(decode_case(8, 2, 64, dtype, 16, "joined", lens, window=window, seed=window), 8, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_softcap_and_scales(dtype):
    c = decode_case(8, 4, 128, dtype, 32, "rows", (5, 200, 77), q_std=6.0)
    _check(c, 8, softcap=20.0)
    _check(c, 8, softcap=0.5, window=64)
    _check(c, 8, scale=0.0)
    _check(c, 8, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens", [
    (32, 8, 128, (5000,)), (4, 1, 64, (20011, 1)), (8, 8, 64, (3, 9000, 0, 1, 4097, 64)),
    (8, 2, 128, tuple([0] * 30 + [700] + [0] * 9)), (8, 2, 128, (33,) * 200), (64, 8, 128, (2500, 10, 2500)),
    (16, 1, 128, (4000, 3, 555)), (8, 2, 256, (3000, 41)),
])
def test_long_and_ragged_batches(dtype, hq, hkv, d, lens):
    _check(decode_case(hq, hkv, d, dtype, 16, "rows", lens, seed=len(lens)), hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,exponents", [(4, (-126, -100)), (4, (-60, 60)), (24, (-40, 40)), (4, (80, 118))])
def test_scales_far_apart(dtype, hq, exponents):
    """Values' scales from one token to the next by up to 2^120: weights keep a reference of their own.  Keys' scales stay
    within what keeps scores finite."""
    c = decode_case(hq, 2, 64, dtype, 16, "rows", (700, 33, 1), seed=3, exponents=exponents)
    gen = torch.Generator(device="cuda").manual_seed(1)
    c["k_scale"][:] = torch.exp2(torch.randint(-9, -5, c["k_scale"].shape, generator=gen, device="cuda").float())
    _check(c, hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_that_are_no_powers_of_two(dtype):
    c = decode_case(8, 2, 128, dtype, 16, "rows", (700, 33, 1), seed=4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for n in ("k_scale", "v_scale"):
        c[n][:] = torch.rand(c[n].shape, generator=gen, device="cuda") * 0.03
    c["v_scale"][c["table"][0, 3].long()] = 0.0  # a row that stands for zeros
    _check(c, 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_of_any_size(dtype):
    """Rows of queries from 2^-60 to 2^60 with keys' scales that undo it, one element far below the others."""
    c = decode_case(12, 6, 64, dtype, 16, "rows", (300, 7), seed=6)
    size = 2.0 ** torch.tensor([-60.0, -20.0, -3.0, 3.0, 20.0, 60.0], device="cuda")
    c["q"] = (c["q"] * size.repeat_interleave(2)[None, :, None].to(c["q"].dtype))
    c["q"][:, :, 5] *= 2.0 ** -20
    c["k_scale"] /= size
    _check(c, 12)
    c["q"][0, 3] = 0
    _check(c, 12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_needles_far_apart_in_magnitude(dtype):
    """Keys' scales rise so that the running maximum does by some 100 several times along the sequence."""
    c = decode_case(4, 2, 64, dtype, 16, "rows", (3000, 3000), seed=4, q_std=1.0)
    table = c["table"].long()
    for i, t in enumerate((0, 17, 700, 1500, 2999)):
        for h in range(2):
            u = c["q"][0, 2 * h].float()
            c["kcache"][table[0, t // 16], t % 16, h] = (u * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            c["k_scale"][table[0, t // 16], t % 16, h] = 2.0 ** (i - 3)
    c["q"][1] *= 20
    _check(c, 4)


def test_queries_as_views_and_without_lse():
    c = decode_case(8, 2, 128, "bf16", 16, "rows", (40, 300, 7))
    ref, _, _ = decode(c, 8)
    wide = torch.full((3, 12 * 128 + 2), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:1 + 8 * 128] = c["q"].reshape(3, -1)
    got, none, err = decode(c, 8, q=wide[:, 1:1 + 8 * 128].unflatten(1, (8, 128)), q_stride=wide.stride(0), lse=False)
    assert err == dck.DCK_OK and none is None and torch.equal(got, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_codes_reach_only_their_heads(dtype):
    c = decode_case(8, 4, 64, dtype, 16, "rows", (100, 100, 1000))
    clean = host(decode(c, 8)[0])
    c["vcache"][c["table"][2, 2].long(), 3, 0, 9] = 0x7f
    c["kcache"][c["table"][2, 50].long(), 3, 3, 9] = 0xff
    c["v_scale"][c["table"][1, 2].long(), 3, 1] = float("inf")
    got, _, err = decode(c, 8)
    assert err == dck.DCK_OK
    got = host(got)
    same = np.ones_like(got, dtype=bool)
    same[2, 0:2, 9] = same[2, 6:8] = same[1, 2:4] = False
    assert np.array_equal(got[same], clean[same])
    assert np.isnan(got[2, 0:2, 9]).all() and np.isnan(got[2, 6:8]).all() and not np.isfinite(got[1, 2:4]).any()


def test_bad_lengths_and_pages_are_recorded_and_give_zeros():
    c = decode_case(8, 2, 64, "bf16", 16, "rows", (40, 300, 7, 90))
    ref = host(decode(c, 8)[0])
    for what in ("negative", "long", "page"):
        d = dict(c, table=c["table"].clone(), seq_len=c["seq_len"].clone())
        if what == "page":
            d["table"][1, 3] = 1 << 20
        else:
            d["seq_len"][1] = -4 if what == "negative" else 301
        out, lse, err = decode(d, 8, max_len=300)
        assert err == dck.DCK_ERR_INVALID
        assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()
        assert np.array_equal(host(out)[[0, 2, 3]], ref[[0, 2, 3]])


def test_calls_repeat_bit_for_bit_in_a_graph_and_on_other_streams():
    c = decode_case(32, 8, 128, "bf16", 16, "rows", (5000, 33, 777, 0))
    cache = dck.QuantCache.from_tensors(c["kcache"], c["k_scale"], c["vcache"], c["v_scale"], 32, "bf16")
    size = dck.dck_quant_decode_workspace_size(cache, 4, 5000)
    ws, out = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.zeros_like(c["q"])
    ref = decode(c, 32)[0]

    def call():
        dck.check(dck.dck_quant_decode_attention(cache, c["q"], 4096, c["kcache"], c["k_scale"], c["vcache"], c["v_scale"],
                                                 c["table"], c["table"].shape[1], c["seq_len"], 4, 5000, 128 ** -0.5, 0, 0.0,
                                                 out, None, ws, size), "dck_quant_decode_attention")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        assert torch.equal(out, ref)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq", [4, 24])
@pytest.mark.parametrize("exponent", [-126, -122, 102])
def test_values_of_the_least_and_largest_scales(dtype, hq, exponent):
    """Values whose powers of two alone are below the least normal number, or as large as the sums may be: 300 tokens of
    values up to 448 2^102 with weights up to 2^8 before the division, 2^8.23 2^8.81 2^102 2^8 < 2^128.  (At 2^119 they are
    not, and outputs were infinite: the interface says how large values may be.)"""
    c = decode_case(hq, 2, 128, dtype, 16, "rows", (1, 40, 300), seed=exponent + 126)
    c["v_scale"].fill_(2.0 ** exponent)
    out, _ = _check(c, hq)
    assert (out != 0).float().mean() > 0.9
