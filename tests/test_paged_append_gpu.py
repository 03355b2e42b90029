"""dck_rope and dck_paged_append against complex multiplications in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import ROPES, TORCH, cache_pair, host

pytestmark = pytest.mark.gpu
POSITIONS = (0, 1, 2, 77, 4095, 4096, 131071, 1 << 20, (1 << 31) - 1)


def _rope(setting):
    kw = dict(setting)
    return dck.Rope(kw.pop("rotary_dim"), kw.pop("theta"), **kw)


def _frequencies(s):
    return P.rope_frequencies(s["rotary_dim"], s["theta"], *[s.get(n, v) for n, v in (
        ("scaling", "none"), ("factor", 1.0), ("slow", 1.0), ("fast", 32.0), ("trained_len", 0))])


def _expected(x, pos, s, transpose=False):
    """(values, bounds): sines and cosines are off by at most 2^-22, the two products and their sum by 2^-23 of their
    magnitudes, the frequency's rounding to a double by pos 2^-53 turns; bf16 rounds once (half an ulp, 2^-8: 7 stored bits)."""
    x = host(x)
    w, layout, mag = _frequencies(s), s.get("layout", "half"), s.get("magnitude", 1.0)
    y = P.rotate(x, pos, w, layout, mag, transpose)
    size = np.abs(x)
    r = 2 * len(w)
    pair = size[..., :r // 2] + size[..., r // 2:r] if layout == "half" else size[..., 0:r:2] + size[..., 1:r:2]
    angle = 2.0 ** -21 + np.asarray(pos, dtype=np.float64)[:, None, None] * 2.0 ** -49 * w
    e = pair * mag * angle
    bound = np.zeros_like(y)
    if layout == "half":
        bound[..., :r // 2] = bound[..., r // 2:r] = e
    else:
        bound[..., 0:r:2] = bound[..., 1:r:2] = e
    return y, bound


def _near(got, want, bound, dtype):
    got = host(got)
    b = bound + np.where(bound > 0, (np.abs(want) + bound) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23), 0)
    assert np.isfinite(got).all() and (np.abs(got - want) <= b).all(), np.max(np.abs(got - want) - b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("setting", ROPES, ids=lambda s: f"{s.get('scaling', 'none')}{s['rotary_dim']}{s.get('layout', 'half')[0]}")
@pytest.mark.parametrize("transpose", [False, True])
def test_rotations(dtype, setting, transpose):
    rng = np.random.default_rng(3)
    for heads, d in ((5, 64), (3, 128), (1, 72)):
        x = torch.from_numpy(rng.standard_normal((len(POSITIONS), heads, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
        pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
        want, bound = _expected(x, POSITIONS, setting, transpose)
        out = torch.full_like(x, float("nan"))
        t = _rope(setting)
        dt = dck.DCK_F32 if dtype == "f32" else dck.DCK_BF16
        dck.check(dck.dck_rope(t, x, len(POSITIONS), heads, d, dt, heads * d, d, pos, out, heads * d, d, transpose), "dck_rope")
        _near(out, want, bound, dtype)
        # views off 16-byte boundaries, heads apart, and in place
        wide = torch.full((len(POSITIONS), heads, d + 3), 7.0, dtype=x.dtype, device="cuda")
        wide[:, :, 1:1 + d] = x
        v = wide[:, :, 1:1 + d]
        dck.check(dck.dck_rope(t, v, len(POSITIONS), heads, d, dt, v.stride(0), v.stride(1), pos, v, v.stride(0), v.stride(1),
                               transpose), "dck_rope")
        torch.cuda.synchronize()
        assert torch.equal(v, out) and (wide[:, :, 0] == 7).all() and (wide[:, :, d + 1:] == 7).all()
        dck.check(dck.dck_rope(t, x, len(POSITIONS), heads, d, dt, heads * d, d, pos, x, heads * d, d, transpose), "dck_rope")
        torch.cuda.synchronize()
        assert torch.equal(x, out)
    assert dck.dck_last_device_error() == dck.DCK_OK


def test_whole_heads_and_many_tokens():
    rng = np.random.default_rng(8)
    for dtype, n, heads, d, s in (("bf16", 1111, 32, 128, dict(rotary_dim=128, theta=1e6)),
                                  ("f32", 517, 7, 256, dict(rotary_dim=256, theta=1e4, layout="interleaved")),
                                  ("bf16", 300, 3, 4096, dict(rotary_dim=256, theta=1e4)),
                                  ("bf16", 2049, 1, 8, dict(rotary_dim=8, theta=1e4)),
                                  ("f32", 1, 64, 128, dict(rotary_dim=64, theta=1e4)),
                                  ("bf16", 9, 129, 64, dict(rotary_dim=48, theta=1e4))):
        x = torch.from_numpy(rng.standard_normal((n, heads, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
        p = rng.integers(0, 200000, n)
        want, bound = _expected(x, p, s)
        out = torch.full_like(x, float("nan"))
        dck.check(dck.dck_rope(_rope(s), x, n, heads, d, dck.DCK_F32 if dtype == "f32" else dck.DCK_BF16, heads * d, d,
                               torch.from_numpy(p.astype(np.int32)).cuda(), out, heads * d, d), "dck_rope")
        _near(out, want, bound, dtype)
        r = s["rotary_dim"]
        assert torch.equal(out[..., r:], x[..., r:])


@pytest.mark.parametrize("setting", ROPES[:5], ids=lambda s: s.get("scaling", "none"))
def test_gradient_against_differences(setting):
    """For L = <g, rope(x)> the call with `transpose` gives dL/dx; central differences of L in random directions agree.
    rope is linear, so a difference's error is rounding alone: 2^-21 per element of rope(x +- u), 2 n elements."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, heads, d = 6, 3, 64
    x, g, u = (torch.randn((n, heads, d), generator=gen, device="cuda") for _ in range(3))
    pos = torch.tensor([0, 5, 100, 5000, 131071, 9], dtype=torch.int32, device="cuda")
    t = _rope(setting)

    def call(v, transpose=False):
        out = torch.empty_like(v)
        dck.check(dck.dck_rope(t, v, n, heads, d, dck.DCK_F32, heads * d, d, pos, out, heads * d, d, transpose), "dck_rope")
        return out.double()
    grad = call(g, True)
    slope = ((call(x + u) - call(x - u)) * g.double()).sum() / 2
    scale = float((call(x).abs() + call(u).abs()).mul(g.abs().double()).sum())
    assert abs(float(slope - (grad * u.double()).sum())) <= 2.0 ** -18 * scale


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("rows", 16), ("joined", 24), ("heads", 1), ("gaps", 100)])
@pytest.mark.parametrize("setting", [ROPES[0], ROPES[4], ROPES[5], None], ids=["half", "yarn", "six", "none"])
@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 128, 1), (6, 6, 64, 45), (5, 1, 72, 700)])
def test_append(dtype, layout, page, setting, hq, hkv, d, n):
    rng = np.random.default_rng(n)
    n_pages = -(-n // page) + 2
    kc, vc = cache_pair(layout, n_pages, page, hkv, d, dtype, fill=3.0)
    qkv = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    if n > 1:
        slots[::7] = -1
    p = rng.integers(0, 100000, n)
    q_out = torch.full((n, hq, d), float("nan"), dtype=qkv.dtype, device="cuda")
    row = qkv.stride(0)
    cache = dck.PagedCache.from_tensors(kc, vc, hq)
    rope = _rope(setting) if setting else None
    args = (row, qkv[:, hq:hq + hkv], row, qkv[:, hq + hkv:], row, n, torch.from_numpy(p.astype(np.int32)).cuda(),
            torch.from_numpy(slots).cuda())
    dck.check(dck.dck_paged_append(cache, rope, qkv[:, :hq], *args, q_out, kc, vc), "dck_paged_append")
    assert dck.dck_last_device_error() == dck.DCK_OK
    s = setting or dict(rotary_dim=2, theta=1.0)
    at = p if setting else np.zeros_like(p)
    q, bq = _expected(qkv[:, :hq], at, s)
    k, bk = _expected(qkv[:, hq:hq + hkv], at, s)
    _near(q_out, q, bq, dtype)
    keep = slots >= 0
    pg, off = torch.from_numpy(slots[keep] // page).cuda(), torch.from_numpy(slots[keep] % page).cuda()
    _near(kc[pg, off], k[keep], bk[keep], dtype)
    assert torch.equal(vc[pg, off], qkv[torch.from_numpy(keep).cuda(), hq + hkv:])
    # nothing else of the caches is touched, gaps between heads and pages included
    for c in (kc, vc):
        c[pg, off] = 3.0
        whole = torch.as_strided(c, (c.untyped_storage().size() // c.element_size(),), (1,), 0)
        if layout != "joined" or c is vc:
            assert (whole == 3).all()
    # keys and values alone
    dck.check(dck.dck_paged_append(cache, rope, None, 0, *args[1:], None, kc, vc), "dck_paged_append")
    torch.cuda.synchronize()
    _near(kc[pg, off], k[keep], bk[keep], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_off_boundaries_and_slots_outside(dtype):
    n, hq, hkv, d = 9, 4, 2, 64
    rng = np.random.default_rng(1)
    wide = torch.from_numpy(rng.standard_normal((n, (hq + 2 * hkv) * d + 5)).astype(np.float32)).to(TORCH[dtype]).cuda()
    kc, vc = cache_pair("rows", 3, 4, hkv, d, dtype, fill=3.0)
    slots = np.array([0, 5, 11, 12, -2, 1 << 40, -1, 7, 3])
    p = rng.integers(0, 1000, n)
    q_out = torch.zeros((n, hq, d), dtype=wide.dtype, device="cuda")
    v3 = lambda a, h: wide[:, a:a + h * d].unflatten(1, (h, d))  # noqa: E731
    q, k, v = v3(1, hq), v3(1 + hq * d, hkv), v3(2 + (hq + hkv) * d, hkv)
    row = wide.stride(0)
    dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(kc, vc, hq), _rope(ROPES[0]), q, row, k, row, v, row, n,
                                   torch.from_numpy(p.astype(np.int32)).cuda(), torch.from_numpy(slots).cuda(), q_out, kc, vc),
              "dck_paged_append")
    assert dck.dck_last_device_error() == dck.DCK_ERR_INVALID
    good = (slots >= 0) & (slots < 12)
    _near(q_out, *_expected(q, p, ROPES[0]), dtype)
    want, bound = _expected(k, p, ROPES[0])
    _near(kc.reshape(12, hkv, d)[slots[good]], want[good], bound[good], dtype)
    assert torch.equal(vc.reshape(12, hkv, d)[slots[good]], v[torch.from_numpy(good).cuda()])
    rest = [s for s in range(12) if s not in slots]
    assert (kc.reshape(12, hkv, d)[rest] == 3).all() and (vc.reshape(12, hkv, d)[rest] == 3).all()


def test_queries_in_place_and_offsets_beyond_32_bits():
    d, page = 128, 16
    n_pages = (1 << 32) // (page * d) + 8
    pool = torch.empty((n_pages, page, 1, d), dtype=torch.bfloat16, device="cuda")
    x = torch.randn((2, 3, d), device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :1].contiguous(), x[:, 1:2].contiguous(), x[:, 2:].contiguous()
    ref = q.clone()
    slots = torch.tensor([(n_pages - 1) * page + 3, 5], dtype=torch.int64, device="cuda")
    pos = torch.tensor([7, 90000], dtype=torch.int32, device="cuda")
    s = dict(rotary_dim=128, theta=1e4)
    for c in (k, v):
        dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(pool, pool, 1), None, None, 0, c, d, c, d, 2, pos, slots,
                                       None, pool, pool), "dck_paged_append")
        torch.cuda.synchronize()
        assert torch.equal(pool[n_pages - 1, 3], c[0]) and torch.equal(pool[0, 5], c[1])
    kc, vc = cache_pair("rows", 2, 16, 1, d, "bf16")
    dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(kc, vc, 1), _rope(s), q, d, k, d, v, d, 2, pos, slots % 16, q,
                                   kc, vc), "dck_paged_append")
    assert dck.dck_last_device_error() == dck.DCK_OK
    _near(q, *_expected(ref, [7, 90000], s), "bf16")


def test_as_many_tokens_as_an_int32_counts():
    n, d = (1 << 31) - 1, 8
    kc, vc = cache_pair("rows", 2, 4, 1, d, "bf16", fill=3.0)
    k, v = (torch.full((1, 1, d), x, dtype=torch.bfloat16, device="cuda") for x in (1.0, 2.0))
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    slots[0], slots[n // 2], slots[n - 1] = 1, 6, 4
    dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(kc, vc, 1), None, None, 0, k, 0, v, 0, n, None, slots, None,
                                   kc, vc), "dck_paged_append")
    assert dck.dck_last_device_error() == dck.DCK_OK
    for c, x in ((kc, 1.0), (vc, 2.0)):
        want = torch.full((8, d), 3.0)
        want[[1, 4, 6]] = x
        assert torch.equal(c.reshape(8, d).float().cpu(), want)
