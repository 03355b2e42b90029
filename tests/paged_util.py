"""Inputs and bounds of the paged cache's tests."""

import numpy as np
import torch

from paper_2607_24331_gb300 import dck

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ROPES = [
    dict(rotary_dim=64, theta=1e4),
    dict(rotary_dim=64, theta=1e6, layout="interleaved", scaling="linear", factor=4.0),
    dict(rotary_dim=32, theta=1e4, scaling="ntk", factor=8.0),
    dict(rotary_dim=64, theta=5e5, scaling="bands", factor=8.0, slow=1.0, fast=4.0, trained_len=8192),
    dict(rotary_dim=64, theta=1e4, layout="interleaved", scaling="yarn", factor=16.0, slow=1.0, fast=32.0,
         trained_len=4096, magnitude=1.2772588722),
    dict(rotary_dim=6, theta=100.0, layout="interleaved"),
    dict(rotary_dim=2, theta=10.0),
]


def cache_pair(layout, n_pages, page, hkv, d, dtype, fill=float("nan")):
    """Key and value caches [n_pages, page, hkv, d] (views), filled with `fill`."""
    kw = dict(dtype=TORCH[dtype], device="cuda")
    if layout == "joined":
        both = torch.full((n_pages, 2, page, hkv, d), fill, **kw)
        return both[:, 0], both[:, 1]
    if layout == "heads":
        return tuple(torch.full((n_pages, hkv, page, d), fill, **kw).transpose(1, 2) for _ in range(2))
    if layout == "gaps":  # strides beyond the rows they hold
        return tuple(torch.full((n_pages, page + 1, hkv + 1, d + 8), fill, **kw)[:, :page, :hkv, :d] for _ in range(2))
    return tuple(torch.full((n_pages, page, hkv, d), fill, **kw) for _ in range(2))


def decode_case(hq, hkv, d, dtype, page, layout, lens, window=0, seed=0, q_std=2.0):
    """Caches that hold NaN wherever a call must not look, table entries outside the pool there."""
    rng = np.random.default_rng(seed)
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 3
    kc, vc = cache_pair(layout, n_pages, page, hkv, d, dtype)
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), max(held) + 2), 2 ** 30, dtype=np.int32)
    table[:, -1] = -5
    at = 0
    for b, n in enumerate(lens):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
        t = torch.arange(max(0, n - window) if window else 0, n)
        if not len(t):
            continue
        p, o = torch.from_numpy(table[b])[t // page].long().cuda(), (t % page).cuda()
        for c in (kc, vc):
            rows = torch.from_numpy(rng.standard_normal((len(t), hkv, d)).astype(np.float32))
            c[p, o] = rows.to(TORCH[dtype]).cuda()
        if window:
            table[b, :(n - window) // page if n > window else 0] = -1
    q = torch.from_numpy(rng.standard_normal((len(lens), hq, d)).astype(np.float32) * q_std).to(TORCH[dtype]).cuda()
    return dict(q=q, kcache=kc, vcache=vc, table=torch.from_numpy(table).cuda(), lens=list(lens),
                seq_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def decode(c, hq, window=0, softcap=0.0, scale=None, max_len=None, lse=True, q=None, q_stride=None, stream=None):
    """(out, lse, device error) of one call; the workspace and outputs hold NaN before it."""
    q = c["q"] if q is None else q
    B, _, d = q.shape
    cache = dck.PagedCache.from_tensors(c["kcache"], c["vcache"], hq)
    max_len = max_len or max(1, max(c["lens"]))
    size = dck.dck_paged_decode_workspace_size(cache, B, max_len)
    ws = torch.full((max(size, 256) // 4 + 1,), float("nan"), device="cuda")
    out = torch.full((B, hq, d), float("nan"), dtype=q.dtype, device="cuda")
    ls = torch.full((B, hq), float("nan"), device="cuda") if lse else None
    dck.check(dck.dck_paged_decode_attention(cache, q, q_stride or hq * d, c["kcache"], c["vcache"], c["table"],
                                             c["table"].stride(0), c["seq_len"], B, max_len,
                                             d ** -0.5 if scale is None else scale, window, softcap, out, ls, ws, size,
                                             stream), "dck_paged_decode_attention")
    err = dck.dck_last_device_error(stream)
    return out, ls, err


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def decode_bounds(dtype, d, n, ref_out, ref_lse, weight, slack, softcap):
    """Bounds of |out - ref| and |lse - ref| from the arithmetic: scores are fp32 sums of d products (each partial sum
    off by at most 2^-22 of the sum of magnitudes, a tensor core's truncation included) and off by a few units of the cap
    through tanh; an error e of all scores changes weights by a factor within exp(+-2e); exponentials, the running
    rescaling and the n-term sums in fp32 add 2^-20 + n 2^-23; with bf16 inputs weights are held as two bf16 (2^-16),
    and the output is rounded once (half an ulp: 2^-8 relative in bf16, which has 7 stored bits)."""
    ds = (d + 8) * 2.0 ** -22 * slack + softcap * 2.0 ** -20
    rel = 2 * ds + 2.0 ** -20 + n[:, None] * 2.0 ** -23 + (2.0 ** -16 if dtype == "bf16" else 0)
    out = weight * rel[..., None] + (np.abs(ref_out) + weight * rel[..., None]) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23)
    lse = ds + 2.0 ** -20 + n[:, None] * 2.0 ** -23 + np.abs(np.where(np.isfinite(ref_lse), ref_lse, 0)) * 2.0 ** -22
    return out, lse
