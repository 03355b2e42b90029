"""Inputs and bounds of the tests of attention over shared prefixes."""

import numpy as np
import torch

import paged_util
import quant_util
from oracle import paged as P
from paged_util import TORCH, cache_pair, host
from paper_2607_24331_gb300 import dck


def shared_case(hq, hkv, d, dtype, quant, page, layout, groups, window=0, seed=0, q_std=2.0):
    """groups: a list of (tokens shared, [length of each row]).  Caches hold NaN wherever a call must not look, tables
    entries outside the pool there.  Rows of a group have the same pages for the tokens they share, whole pages or (rows
    that have nothing beyond) a part of the last one."""
    rng = np.random.default_rng(seed)
    rows = [n for _, lens in groups for n in lens]
    width = -(-max(rows + [1]) // page) + 2
    table = np.full((len(rows), width), 2 ** 30, dtype=np.int64)
    n_pages, b, fill = 0, 0, []  # fill: (row, tokens) written by that row's table
    for share, lens in groups:
        longest = max(lens)
        common = min(share, longest) if len(lens) > 1 else 0
        assert common % page == 0 or common == longest
        whole = -(-common // page)
        for i, n in enumerate(lens):
            mine = -(-n // page)
            if len(lens) > 1:
                table[b, :min(whole, mine)] = n_pages + np.arange(min(whole, mine))
            at = min(whole, mine) if len(lens) > 1 else 0
            table[b, at:mine] = n_pages + whole + sum(max(0, -(-m // page) - whole) for m in lens[:i]) + np.arange(mine - at)
            first = max(0, n - window) if window else 0
            fill.append((b, np.arange(first, n)))
            b += 1
        n_pages += whole + sum(max(0, -(-m // page) - whole) for m in lens)
    n_pages += 3
    perm = rng.permutation(n_pages)
    real = table < 2 ** 30
    table[real] = perm[table[real]]
    c = dict(lens=rows, dtype=dtype, quant=quant)
    if quant:
        c["kcache"], c["k_scale"], c["vcache"], c["v_scale"] = quant_util.code_pair(layout, n_pages, page, hkv, d)
    else:
        c["kcache"], c["vcache"] = cache_pair(layout, n_pages, page, hkv, d, dtype)
    for b, t in fill:
        if not len(t):
            continue
        p, o = torch.from_numpy(table[b][t // page]).cuda(), torch.from_numpy(t % page).cuda()
        for k, s in (("kcache", "k_scale"), ("vcache", "v_scale")):
            if quant:
                codes, scales = quant_util.rows_of(rng, len(t), hkv, d)
                c[k][p, o], c[s][p, o] = codes.cuda(), scales.cuda()
            else:
                c[k][p, o] = torch.from_numpy(rng.standard_normal((len(t), hkv, d)).astype(np.float32)).to(TORCH[dtype]).cuda()
    c["q"] = torch.from_numpy(rng.standard_normal((len(rows), hq, d)).astype(np.float32) * q_std).to(TORCH[dtype]).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    c["table"] = torch.from_numpy(table.astype(np.int32)).cuda()
    c["seq_len"] = torch.tensor(rows, **i32)
    c["group_start"] = torch.tensor(np.cumsum([0] + [len(g[1]) for g in groups]), **i32)
    c["shared_len"] = torch.tensor([g[0] for g in groups], **i32)
    c["max_own"] = max([1] + [n - (min(n, g[0]) if len(g[1]) > 1 else 0) for g in groups for n in g[1]])
    return c


def attend(c, hq, window=0, softcap=0.0, scale=None, max_len=None, max_own=None, lse=True, q=None, q_stride=None, stream=None):
    """(out, lse, device error) of one call; the workspace and outputs hold NaN before it."""
    q = c["q"] if q is None else q
    B, _, d = q.shape
    max_len, max_own = max_len or max(1, max(c["lens"])), max_own or c["max_own"]
    if c["quant"]:
        caches = (c["kcache"], c["k_scale"], c["vcache"], c["v_scale"])
        cache, call = dck.QuantCache.from_tensors(*caches, hq, c["dtype"]), dck.dck_quant_shared_attention
        size = dck.dck_quant_shared_workspace_size(cache, B, max_len, max_own)
    else:
        caches = (c["kcache"], c["vcache"])
        cache, call = dck.PagedCache.from_tensors(*caches, hq), dck.dck_paged_shared_attention
        size = dck.dck_paged_shared_workspace_size(cache, B, max_len, max_own)
    ws = torch.full((max(size, 256) // 4 + 1,), float("nan"), device="cuda")
    out = torch.full((B, hq, d), float("nan"), dtype=q.dtype, device="cuda")
    ls = torch.full((B, hq), float("nan"), device="cuda") if lse else None
    dck.check(call(cache, q, q_stride or hq * d, *caches, c["table"], c["table"].stride(0), c["seq_len"], B, max_len, max_own,
                   c["group_start"].numel() - 1, c["group_start"], c["shared_len"], d ** -0.5 if scale is None else scale, window,
                   softcap, out, ls, ws, size, stream), "shared attention")
    err = dck.dck_last_device_error(stream)
    return out, ls, err


def bounds(c, d, n, ref, rlse, weight, slack, softcap):
    """As for calls by single rows, with the weights of the shared part in one term where a tile has more than 8 queries:
    half a step of bf16 (2^-8) on bf16 caches, of fp16 (2^-11) on 8-bit ones."""
    if c["quant"]:
        most = float(np.nan_to_num(c["v_scale"].cpu().numpy().astype(np.float64), nan=0.0).max())
        bo, bl = quant_util.decode_bounds(c["dtype"], 16, d, n, ref, rlse, weight, slack, softcap, most)
    else:
        bo, bl = paged_util.decode_bounds(c["dtype"], d, n, ref, rlse, weight, slack, softcap)
        if c["dtype"] == "bf16":
            bo = bo + weight * 2.0 ** -8
    return bo, bl


def check(c, hq, window=0, softcap=0.0, scale=None, rows=None, expect=dck.DCK_OK, **kw):
    """The call against the plain definition, row by row (`rows`: those to look at; `expect`: the device error)."""
    out, lse, err = attend(c, hq, window, softcap, scale, **kw)
    assert err == expect
    rows = np.arange(len(c["lens"])) if rows is None else np.asarray(rows)
    d = c["q"].shape[2]
    scale = float(np.float32(d ** -0.5 if scale is None else scale))
    k, v = ((quant_util.values(c), quant_util.values(c, "vcache", "v_scale")) if c["quant"] else (host(c["kcache"]), host(c["vcache"])))
    lens = np.asarray(c["lens"])[rows]
    ref, rlse, weight, slack = P.paged_decode(host(c["q"])[rows], k, v, c["table"].cpu().numpy()[rows], lens, scale, window, softcap)
    n = np.minimum(lens, window or max(c["lens"])).astype(np.float64)
    bo, bl = bounds(c, d, n, ref, rlse, weight, slack, softcap)
    got, glse = host(out)[rows], host(lse)[rows]
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bo).all(), np.max(np.abs(got - ref) - bo)
    assert np.array_equal(np.isneginf(glse), np.isneginf(rlse))
    f = np.isfinite(rlse)
    assert (np.abs(glse[f] - rlse[f]) <= bl[f]).all(), np.max(np.abs(glse[f] - rlse[f]) - bl[f])
    return out, lse
