"""dck_rope and dck_paged_append at positions below zero (keys turned back by a distance), against complex
multiplications in 64 bits: both layouts, whole rows in vectors and single elements, and the transpose."""

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import ROPES, TORCH, cache_pair
from test_paged_append_gpu import _expected, _frequencies, _near, _rope

pytestmark = pytest.mark.gpu
POSITIONS = (-1, -2, -5, -1000, -4096, -131072, -(1 << 31) + 1, -(1 << 31), 0, 7, (1 << 31) - 1)
SETTINGS = ROPES + [dict(rotary_dim=64, theta=1e4, layout="interleaved"), dict(rotary_dim=24, theta=1e4)]


def _at(x, pos, s, transpose=False):
    """Values at the positions; bounds depend on the positions' size alone."""
    _, bound = _expected(x, np.abs(np.asarray(pos, dtype=np.int64)), s, transpose)
    return P.rotate(x.float().cpu().numpy().astype(np.float64), pos, _frequencies(s), s.get("layout", "half"),
                    s.get("magnitude", 1.0), transpose), bound


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("setting", SETTINGS, ids=lambda s: f"{s.get('scaling', 'none')}{s['rotary_dim']}{s.get('layout', 'half')[0]}")
@pytest.mark.parametrize("transpose", [False, True])
def test_rotations(dtype, setting, transpose):
    rng = np.random.default_rng(5)
    n = len(POSITIONS)
    t, dt = _rope(setting), dck.DCK_F32 if dtype == "f32" else dck.DCK_BF16
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
    for heads, d in ((5, 64), (1, 72)):
        x = torch.from_numpy(rng.standard_normal((n, heads, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
        want, bound = _at(x, POSITIONS, setting, transpose)
        out = torch.full_like(x, float("nan"))
        dck.check(dck.dck_rope(t, x, n, heads, d, dt, heads * d, d, pos, out, heads * d, d, transpose), "dck_rope")
        _near(out, want, bound, dtype)
        wide = torch.zeros((n, heads, d + 3), dtype=x.dtype, device="cuda")  # rows off 16-byte boundaries
        wide[:, :, 1:1 + d] = x
        v = wide[:, :, 1:1 + d]
        out = torch.full_like(x, float("nan"))
        dck.check(dck.dck_rope(t, v, n, heads, d, dt, v.stride(0), v.stride(1), pos, out, heads * d, d, transpose), "dck_rope")
        _near(out, want, bound, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("setting", [ROPES[0], ROPES[4], ROPES[5]], ids=["half", "yarn", "six"])
def test_append(dtype, setting):
    rng = np.random.default_rng(6)
    n, hq, hkv, d = len(POSITIONS), 4, 2, 64
    kc, vc = cache_pair("rows", 2, 16, hkv, d, dtype, fill=3.0)
    qkv = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
    slots = torch.from_numpy(rng.permutation(32)[:n].astype(np.int64)).cuda()
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
    q_out, row = torch.full((n, hq, d), float("nan"), dtype=qkv.dtype, device="cuda"), qkv.stride(0)
    dck.check(dck.dck_paged_append(dck.PagedCache.from_tensors(kc, vc, hq), _rope(setting), qkv, row, qkv[:, hq:], row,
                                   qkv[:, hq + hkv:], row, n, pos, slots, q_out, kc, vc), "dck_paged_append")
    assert dck.dck_last_device_error() == dck.DCK_OK
    _near(q_out, *_at(qkv[:, :hq], POSITIONS, setting), dtype)
    _near(kc.reshape(32, hkv, d)[slots], *_at(qkv[:, hq:hq + hkv], POSITIONS, setting), dtype)
    assert torch.equal(vc.reshape(32, hkv, d)[slots], qkv[:, hq + hkv:])
