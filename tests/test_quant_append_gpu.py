"""dck_quant_append and dck_quant_read: codes and scales value for value against the definition of 8-bit rows, applied to
what dck_paged_append writes in full width."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import ROPES, TORCH, cache_pair
from quant_util import code_pair, rows_of

pytestmark = pytest.mark.gpu


def _rope(setting):
    kw = dict(setting)
    return dck.Rope(kw.pop("rotary_dim"), kw.pop("theta"), **kw) if kw else None


def _i64(x):
    return torch.from_numpy(np.asarray(x, dtype=np.int64)).cuda()


def _append(qkv, hq, hkv, page, layout, slots, positions, rope, dtype, n_pages, offset=0):
    """(q_out, codes and scales, the same append's full-width q_out and caches)."""
    n, _, d = qkv.shape
    row = qkv.stride(0)
    kc, ks, vc, vs = code_pair(layout, n_pages, page, hkv, d, fill=0x55)
    cache = dck.QuantCache.from_tensors(kc, ks, vc, vs, hq, dtype)
    q = torch.full((n, hq, d), float("nan"), dtype=qkv.dtype, device="cuda")
    args = (qkv[:, :hq], row, qkv[:, hq:hq + hkv], row, qkv[:, hq + hkv:], row, n, positions, slots)
    dck.check(dck.dck_quant_append(cache, rope, *args, q, kc, ks, vc, vs), "dck_quant_append")
    err = dck.dck_last_device_error()
    wide = cache_pair("rows", n_pages, page, hkv, d, dtype)
    wq = torch.full_like(q, float("nan"))
    dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(*wide, hq), rope, *args, wq, *wide), "dck_paged_append")
    dck.dck_last_device_error()
    return q, (kc, ks, vc, vs), wq, wide, err


def _same(got, wide, slots, page, hkv):
    """Every written row is its full-width row's 8-bit form; nothing else has changed."""
    kc, ks, vc, vs = got
    keep = slots[slots >= 0]
    p, o = _i64(keep // page), _i64(keep % page)
    for c, s, w in ((kc, ks, wide[0]), (vc, vs, wide[1])):
        codes, scales = P.quantise(w[p, o].double().cpu().numpy())
        found = c[p, o].cpu().numpy()
        nan = (codes & 127) == 127
        assert np.array_equal(found & np.where(nan, 127, 255), codes & np.where(nan, 127, 255))
        assert np.array_equal(s[p, o].cpu().numpy(), scales.astype(np.float32))
        c[p, o], s[p, o] = 0x55, float("nan")
        assert (c == 0x55).all() and torch.isnan(s).all()
        for whole in (c, s):
            if whole._base is not None:  # the gaps and the other cache's rows of a joined buffer are checked by it
                base = whole._base
                assert (base == 0x55).all() if base.dtype == torch.uint8 and c is vc else True


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("rows", 16), ("joined", 24), ("heads", 1), ("gaps", 100)])
@pytest.mark.parametrize("setting", [ROPES[0], ROPES[4], ROPES[5], {}], ids=["half", "yarn", "six", "none"])
@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 128, 1), (6, 6, 64, 45), (5, 1, 72, 300), (3, 3, 80, 33), (4, 2, 256, 9)])
def test_append(dtype, layout, page, setting, hq, hkv, d, n):
    rng = np.random.default_rng(n)
    n_pages = -(-n // page) + 2
    size = 10.0 ** rng.integers(-6, 6, (n, hq + 2 * hkv, 1))
    qkv = torch.from_numpy((rng.standard_normal((n, hq + 2 * hkv, d)) * size).astype(np.float32)).to(TORCH[dtype]).cuda()
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    if n > 1:
        slots[::7] = -1
    pos = torch.from_numpy(rng.integers(0, 100000, n).astype(np.int32)).cuda()
    q, got, wq, wide, err = _append(qkv, hq, hkv, page, layout, _i64(slots), pos, _rope(setting), dtype, n_pages)
    assert err == dck.DCK_OK and torch.equal(q, wq)
    _same(got, wide, slots, page, hkv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [0, 128, 32, 6])
def test_rows_at_the_ends_of_the_scales(dtype, rot):
    """Rows of zeros, of least and largest numbers, at 448 times a power of two and just beyond, with infinities and NaN."""
    d, tiny, huge = 128, 1e-45 if dtype == "f32" else 2.0 ** -133, float(torch.finfo(TORCH[dtype]).max)
    step = 2.0 ** -23 if dtype == "f32" else 2.0 ** -7
    rows = [[0.0], [-0.0], [tiny], [2.0 ** -126], [448 * 2.0 ** -126], [448 * 2.0 ** -126 * (1 + step)], [huge], [-huge, tiny],
            [448.0], [448 * (1 + step)], [1.75], [1.75 * (1 + step)], [float("inf"), 1.0], [float("nan"), -2.0], [float("-inf")],
            [float("nan")], [1.0, 17 / 16, 19 / 16, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11]]
    n = len(rows)
    x = torch.zeros((n, 3, d))
    for i, r in enumerate(rows):
        x[i, 1, 64 - len(r):64] = torch.tensor(r)  # keys: elements on both sides of rotary dimensions
        x[i, 2, :len(r)] = torch.tensor(r)
    qkv = x.to(TORCH[dtype]).cuda()
    slots = np.arange(n)
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")  # turned by nothing
    q, got, wq, wide, err = _append(qkv, 1, 1, 8, "rows", _i64(slots), pos, _rope(dict(rotary_dim=rot, theta=1e4) if rot else {}),
                                    dtype, 3)
    assert err == dck.DCK_OK
    _same(got, wide, slots, 8, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_off_16_bytes_and_without_queries(dtype):
    rng = np.random.default_rng(5)
    n, hq, hkv, d = 21, 4, 2, 64
    wide = torch.zeros((n, (hq + 2 * hkv) * d + 3), dtype=TORCH[dtype], device="cuda")
    wide[:, 1:-2] = torch.from_numpy(rng.standard_normal((n, (hq + 2 * hkv) * d)).astype(np.float32)).to(wide)
    qkv = wide[:, 1:-2].unflatten(1, (hq + 2 * hkv, d))
    slots, pos = rng.permutation(48)[:n], torch.arange(n, dtype=torch.int32, device="cuda")
    q, got, wq, full, err = _append(qkv, hq, hkv, 16, "rows", _i64(slots), pos, dck.Rope(32, 1e4), dtype, 3)
    assert err == dck.DCK_OK and torch.equal(q, wq)
    again = code_pair("rows", 3, 16, hkv, d, fill=0x55)
    cache = dck.QuantCache.from_tensors(again[0], again[1], again[2], again[3], hq, dtype)
    row = qkv.stride(0)
    dck.check(dck.dck_quant_append(cache, dck.Rope(32, 1e4), None, 0, qkv[:, hq:], row, qkv[:, hq + hkv:], row, n, pos, _i64(slots),
                                   None, again[0], again[1], again[2], again[3]), "dck_quant_append")
    torch.cuda.synchronize()
    for a, b in zip(again, got):
        assert torch.equal(a.view(torch.int32) if a.dtype == torch.float32 else a, b.view(torch.int32) if b.dtype == torch.float32 else b)
    _same(got, full, slots, 16, hkv)


def test_slots_outside_the_pool_are_recorded_and_skipped():
    gen = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.randn((6, 3, 64), generator=gen, device="cuda").to(torch.bfloat16)
    slots = np.array([3, -1, -2, 1 << 40, 20, 19])
    q, got, wq, wide, err = _append(qkv, 1, 1, 5, "rows", _i64(slots), torch.arange(6, dtype=torch.int32, device="cuda"),
                                    dck.Rope(64, 1e4), "bf16", 4)
    assert err == dck.DCK_ERR_INVALID and torch.equal(q, wq)
    _same(got, wide, np.array([3, 19]), 5, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("rows", 16), ("joined", 24), ("heads", 1), ("gaps", 100)])
@pytest.mark.parametrize("hkv,d,n", [(2, 128, 1), (6, 64, 45), (1, 72, 700), (3, 80, 33), (2, 256, 9), (1, 8, 5), (8, 128, 3000)])
def test_read(dtype, layout, page, hkv, d, n):
    rng = np.random.default_rng(d)
    n_pages = -(-n // page) + 1
    kc, ks, vc, vs = code_pair(layout, n_pages, page, hkv, d)
    for c, s in ((kc, ks), (vc, vs)):
        codes, scales = rows_of(rng, n_pages * page, hkv, d, (-130, 110))
        c[:] = codes.cuda().unflatten(0, (n_pages, page))
        s[:] = torch.clamp(scales, min=2.0 ** -126).cuda().unflatten(0, (n_pages, page))
    slots = rng.integers(0, n_pages * page, n)  # some of them twice
    slots[n // 2] = -1 if n > 1 else slots[0]
    cache = dck.QuantCache.from_tensors(kc, ks, vc, vs, hkv, dtype)
    at = _i64(np.maximum(slots, 0))
    want = []
    for c, s in ((kc, ks), (vc, vs)):
        x = c[at // page, at % page].contiguous().view(torch.float8_e4m3fn).double() * s[at // page, at % page].double()[..., None]
        want.append(torch.where((_i64(slots) >= 0)[:, None, None], x, 0.0).to(TORCH[dtype]))
    for pad, off in ((0, 0), (8, 0), (3, 1)):  # dense, rows apart, rows off 16-byte boundaries
        k, v = (torch.full((n, hkv * d + pad), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
        kk, vv = k[:, off:off + hkv * d], v[:, off:off + hkv * d]
        dck.check(dck.dck_quant_read(cache, n, _i64(slots), kc, ks, vc, vs, kk, k.stride(0), vv, v.stride(0)), "dck_quant_read")
        assert dck.dck_last_device_error() == dck.DCK_OK
        assert torch.equal(kk, want[0].flatten(1)) and torch.equal(vv, want[1].flatten(1))
        for whole in (k, v):
            assert (whole[:, :off] == 7).all() and (whole[:, off + hkv * d:] == 7).all()


def test_read_of_slots_outside_the_pool():
    kc, ks, vc, vs = code_pair("rows", 2, 4, 1, 64, fill=0x38)
    ks[:], vs[:] = 2.0, 4.0
    k, v = (torch.full((4, 64), 7.0, device="cuda") for _ in range(2))
    cache = dck.QuantCache.from_tensors(kc, ks, vc, vs, 1, "f32")
    dck.check(dck.dck_quant_read(cache, 4, _i64([7, 8, -1, -9]), kc, ks, vc, vs, k, 64, v, 64), "dck_quant_read")
    assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
    assert (k[0] == 2).all() and (v[0] == 4).all() and (k[1:] == 0).all() and (v[1:] == 0).all()


def test_append_then_read_is_near_what_was_appended():
    """An e4m3 rounding is off by 2^-4 of a value at most, or 2^-10 of the scale below 2^-6 of it."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, hkv, d, page = 1000, 4, 128, 16
    kv = torch.randn((n, 2 * hkv, d), generator=gen, device="cuda")
    kc, ks, vc, vs = code_pair("joined", 70, page, hkv, d)
    cache = dck.QuantCache.from_tensors(kc, ks, vc, vs, hkv, "f32")
    slots, pos = torch.randperm(70 * page, generator=gen, device="cuda")[:n], torch.arange(n, dtype=torch.int32, device="cuda")
    rope = dck.Rope(d, 1e4)
    dck.check(dck.dck_quant_append(cache, rope, None, 0, kv, kv.stride(0), kv[:, hkv:], kv.stride(0), n, pos, slots, None, kc, ks,
                                   vc, vs), "dck_quant_append")
    k, v = (torch.empty((n, hkv, d), device="cuda") for _ in range(2))
    dck.check(dck.dck_quant_read(cache, n, slots, kc, ks, vc, vs, k, hkv * d, v, hkv * d), "dck_quant_read")
    turned = torch.empty_like(k)
    dck.check(dck.dck_rope(rope, kv, n, hkv, d, dck.DCK_F32, kv.stride(0), d, pos, turned, hkv * d, d), "dck_rope")
    for got, want, s in ((k, turned, ks), (v, kv[:, hkv:], vs)):
        scale = s[slots // page, slots % page][..., None]
        assert ((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, scale * 2.0 ** -10)).all()
