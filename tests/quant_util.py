"""Inputs and bounds of the 8-bit cache's tests."""

import numpy as np
import torch

from oracle import paged as P
from paged_util import TORCH, cache_pair
from paper_2607_24331_gb300 import dck


def code_pair(layout, n_pages, page, hkv, d, fill=0x7f):
    """Code caches and scales [n_pages, page, hkv, ...] (views), codes filled with `fill` (NaN), scales with NaN."""
    def scales():
        kw = dict(device="cuda")
        if layout == "joined":
            both = torch.full((n_pages, 2, page, hkv), float("nan"), **kw)
            return both[:, 0], both[:, 1]
        if layout == "heads":
            return tuple(torch.full((n_pages, hkv, page), float("nan"), **kw).transpose(1, 2) for _ in range(2))
        if layout == "gaps":
            return tuple(torch.full((n_pages, page + 1, hkv + 3), float("nan"), **kw)[:, :page, :hkv] for _ in range(2))
        return tuple(torch.full((n_pages, page, hkv), float("nan"), **kw) for _ in range(2))
    wide = -(-d // 16) * 16  # strides are multiples of 16 bytes
    if layout == "gaps":
        codes = [torch.full((n_pages, page + 1, hkv + 1, wide + 16), fill, dtype=torch.uint8, device="cuda")[:, :page, :hkv, :d]
                 for _ in range(2)]
    elif layout == "joined":
        both = torch.full((n_pages, 2, page, hkv, wide), fill, dtype=torch.uint8, device="cuda")
        codes = [both[:, 0, ..., :d], both[:, 1, ..., :d]]
    elif layout == "heads":
        codes = [torch.full((n_pages, hkv, page, wide), fill, dtype=torch.uint8, device="cuda").transpose(1, 2)[..., :d]
                 for _ in range(2)]
    else:
        codes = [torch.full((n_pages, page, hkv, wide), fill, dtype=torch.uint8, device="cuda")[..., :d] for _ in range(2)]
    k, v = scales()
    return codes[0], k, codes[1], v


def rows_of(rng, n, hkv, d, exponents=(-8, -5)):
    """Codes (magnitudes up to 448, of a normal distribution) and scales of n tokens."""
    x = np.clip(rng.standard_normal((n, hkv, d)) * 120, -448, 448)
    codes = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, torch.from_numpy(2.0 ** rng.integers(*exponents, (n, hkv))).float()


def decode_case(hq, hkv, d, dtype, page, layout, lens, window=0, seed=0, q_std=2.0, exponents=(-8, -5)):
    """Caches that hold NaN wherever a call must not look, table entries outside the pool there."""
    rng = np.random.default_rng(seed)
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 3
    kc, ks, vc, vs = code_pair(layout, n_pages, page, hkv, d)
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), max(held) + 2), 2 ** 30, dtype=np.int32)
    table[:, -1] = -5
    at = 0
    for b, n in enumerate(lens):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
        t = np.arange(max(0, n - window) if window else 0, n)
        if not len(t):
            continue
        p, o = torch.from_numpy(table[b][t // page]).long().cuda(), torch.from_numpy(t % page).cuda()
        for c, s in ((kc, ks), (vc, vs)):
            codes, scales = rows_of(rng, len(t), hkv, d, exponents)
            c[p, o], s[p, o] = codes.cuda(), scales.cuda()
        if window:
            table[b, :(n - window) // page if n > window else 0] = -1
    q = torch.from_numpy(rng.standard_normal((len(lens), hq, d)).astype(np.float32) * q_std).to(TORCH[dtype]).cuda()
    return dict(q=q, kcache=kc, k_scale=ks, vcache=vc, v_scale=vs, table=torch.from_numpy(table).cuda(), lens=list(lens),
                seq_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), dtype=dtype)


def decode(c, hq, window=0, softcap=0.0, scale=None, max_len=None, lse=True, q=None, q_stride=None, stream=None):
    """(out, lse, device error) of one call; the workspace and outputs hold NaN before it."""
    q = c["q"] if q is None else q
    B, _, d = q.shape
    cache = dck.QuantCache.from_tensors(c["kcache"], c["k_scale"], c["vcache"], c["v_scale"], hq, c["dtype"])
    max_len = max_len or max(1, max(c["lens"]))
    size = dck.dck_quant_decode_workspace_size(cache, B, max_len)
    ws = torch.full((max(size, 256) // 4 + 1,), float("nan"), device="cuda")
    out = torch.full((B, hq, d), float("nan"), dtype=q.dtype, device="cuda")
    ls = torch.full((B, hq), float("nan"), device="cuda") if lse else None
    dck.check(dck.dck_quant_decode_attention(cache, q, q_stride or hq * d, c["kcache"], c["k_scale"], c["vcache"],
                                             c["v_scale"], c["table"], c["table"].stride(0), c["seq_len"], B, max_len,
                                             d ** -0.5 if scale is None else scale, window, softcap, out, ls, ws, size,
                                             stream), "dck_quant_decode_attention")
    err = dck.dck_last_device_error(stream)
    return out, ls, err


def values(c, k="kcache", s="k_scale"):
    return P.stand_for(c[k].cpu().numpy(), c[s].cpu().numpy())


def decode_bounds(dtype, qpg, d, n, ref_out, ref_lse, weight, slack, softcap, most):
    """Bounds of |out - ref| and |lse - ref| from the arithmetic, as for the other caches (paged_util.decode_bounds: fp32
    scores, exponentials, sums and the output's rounding), and: fp32 queries in two fp16 terms (2^-22 of each product);
    weights in two fp16 terms (2^-22), or one of bf16 calls with more than 8 queries on a KV head (half a step of fp16:
    2^-11), and of each weight an error of 2^-32 of the largest at least (half of fp16's least step, 2^-25, of a largest
    weight of 2^7), which multiplies codes up to 448 of scale `most`."""
    ds = (d + 10) * 2.0 ** -22 * slack + softcap * 2.0 ** -20
    one = dtype == "bf16" and qpg > 8
    rel = 2 * ds + 2.0 ** -20 + n[:, None] * 2.0 ** -23 + (2.0 ** -11 if one else 2.0 ** -22)
    out = weight * rel[..., None] + (n[:, None] * 2.0 ** -32 * 448 * most)[..., None]
    out = out + (np.abs(ref_out) + out) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23)
    lse = ds + 2.0 ** -20 + n[:, None] * 2.0 ** -23 + np.abs(np.where(np.isfinite(ref_lse), ref_lse, 0)) * 2.0 ** -22
    return out, lse
