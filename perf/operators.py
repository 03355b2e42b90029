"""The paged key-value cache's operators, as cases to be timed and compared.

Every case is one call of a public entry point of ``dck``, or the same in elementary
torch operations.  Kinds:

  pages   dck_page_update: block tables, free list and slot map from request lengths
  rope    dck_rope: rotary positions, or their transpose (the gradient)
  append  dck_paged_append: new tokens' queries rotated, keys rotated and written with
          the values into their cache rows
  attend  dck_paged_decode_attention: one query per sequence over the pages

Lengths are ``lo == hi`` (all alike) or ragged, drawn log-uniformly from [lo, hi] with
``lens_seed``; ``idle`` of the sequences are empty (the padding of a captured batch).
Cache ``layout``: "rows" [pages, page, heads, d], keys and values apart; "joined" one buffer
[pages, 2, page, heads, d]; "heads" [pages, heads, page, d].
"""

import math
import random

import torch

own = False

# (query heads, KV heads, head dim)
HEADS = {
    "mha32": (32, 32, 128),  # the repository's 32-head layer
    "gqa8": (32, 8, 128),    # its layers with 8 KV heads
    "mha8": (8, 8, 64),      # its small fp32 layer
    "mqa": (16, 1, 128),     # one KV head for all queries
    "odd": (10, 2, 80),      # a head dim that is no power of two
    "wide": (8, 2, 256),     # the widest head
}

# rotary settings: (rotary share of the head, theta, layout, scaling, factor, a, b, trained length, magnitude)
ROPES = {
    "plain": (1.0, 1e4, "half", "none", 1.0, 0.0, 0.0, 0, 1.0),
    "linear": (1.0, 1e6, "half", "linear", 4.0, 0.0, 0.0, 0, 1.0),
    "ntk": (1.0, 1e4, "interleaved", "ntk", 8.0, 0.0, 0.0, 0, 1.0),
    "bands": (1.0, 5e5, "half", "bands", 8.0, 1.0, 4.0, 8192, 1.0),
    "yarn": (1.0, 1e4, "half", "yarn", 16.0, 1.0, 32.0, 4096, 1.2772588722),
    "part": (0.5, 1e4, "interleaved", "none", 1.0, 0.0, 0.0, 0, 1.0),
}


def _case(name, kind, **kw):
    c = dict(kind=kind, heads="gqa8", f32=False, batch=1, lo=1, hi=1, idle=0, page=16, layout="rows", window=0,
             softcap=0.0, tokens=0, rope="plain", transpose=False, spare=0, lens_seed=1)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the page bookkeeping of one decode step of a small batch: latency
        _case("pages-b16-step", "pages", batch=16, lo=100, hi=4096, tokens=1, spare=64),
        # a busy scheduler's step: prompts admitted, finished requests released, most others one token on
        _case("pages-b256-mixed", "pages", batch=256, lo=64, hi=8192, tokens=128, spare=20000, lens_seed=5),
        # queries of one decode step of the small fp32 layer, half of each head rotated
        _case("rope-f32-b8-part", "rope", heads="mha8", f32=True, tokens=8, rope="part"),
        # the gradient through the rotation of a training batch's queries, context-extended positions
        _case("rope-bf16-16384-grad", "rope", heads="mha32", tokens=16384, rope="yarn", transpose=True),
        # one user's new token: latency
        _case("append-b1", "append", heads="gqa8", tokens=1, rope="bands"),
        # a serving batch's new tokens, into a joined cache
        _case("append-b48", "append", heads="mha32", tokens=48, layout="joined", page=32),
        # a long prompt pair of 2 x 8192 tokens
        _case("append-16384", "append", heads="gqa8", tokens=16384, page=64, rope="bands"),
        # one user in a short conversation: latency
        _case("attend-gqa-b1-777", "attend", heads="gqa8", batch=1, lo=777, hi=777),
        # the small fp32 layer, a few users
        _case("attend-f32-b4-512", "attend", heads="mha8", f32=True, batch=4, lo=300, hi=512, page=24),
        # the ordinary serving batch on the 32-head layer
        _case("attend-mha-b16-4096", "attend", heads="mha32", batch=16, lo=4096, hi=4096, page=32),
        # a continuous batch, every sequence of another length, some slots idle
        _case("attend-gqa-b32-ragged", "attend", heads="gqa8", batch=32, lo=1024, hi=16384, idle=3, layout="joined"),
        # the longest contexts: two documents of 128k tokens
        _case("attend-gqa-b2-131072", "attend", heads="gqa8", batch=2, lo=131072, hi=131072, page=64, layout="heads"),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MAX_CACHE = 2 * 131072 * 8 * 128  # key elements of an attend call, padded to its longest sequence


def draw(rng):
    kind = rng.choice(("pages", "rope", "append", "attend", "attend", "attend"))
    seed = rng.randrange(1 << 20)
    page = rng.choice((1, 8, 16, 16, 24, 32, 64, 100, 128, 256))
    layout = rng.choice(("rows", "joined", "heads"))
    rope = rng.choice(sorted(ROPES))
    f32 = rng.random() < 0.25
    heads = rng.choice(("mha32", "gqa8", "gqa8", "mha8", "mqa", "odd", "wide"))
    if kind == "pages":
        batch = _logint(rng, 1, 1024)
        hi = _logint(rng, 16, 16384 if batch <= 256 else 2048)
        return _case(None, kind, batch=batch, lo=max(1, hi // 32), hi=hi, page=max(page, 8),
                     tokens=_logint(rng, 1, max(1, min(hi, 16384 // batch))), spare=_logint(rng, 1, 16384), lens_seed=seed)
    if kind in ("rope", "append"):
        hq, _, d = HEADS[heads]
        most = 16384 * 32 * 128 // (hq * d) // (2 if f32 else 1)
        return _case(None, kind, heads=heads, f32=f32, tokens=_logint(rng, 1, min(16384, most)), page=page, layout=layout,
                     rope=rope, transpose=kind == "rope" and rng.random() < 0.5, lens_seed=seed)
    _, hkv, d = HEADS[heads]
    while True:
        batch, hi = _logint(rng, 1, 128), _logint(rng, 1, 131072)
        if batch * hi * hkv * d * (2 if f32 else 1) <= MAX_CACHE:
            break
    return _case(None, kind, heads=heads, f32=f32, batch=batch, lo=rng.choice((hi, max(1, hi // 16))), hi=hi,
                 idle=rng.choice((0, 0, batch // 8)), page=page, layout=layout,
                 window=rng.choice((0, 0, 0, _logint(rng, 1, 4096))), softcap=rng.choice((0.0, 0.0, 30.0)), lens_seed=seed)


def _lens(case):
    rng = random.Random(case["lens_seed"])
    lens = [_logint(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    for b in rng.sample(range(case["batch"]), case["idle"]):
        lens[b] = 0
    return lens


def _page_lens(case):
    """Lengths before and after a scheduler's step: most requests take one token (or a few, with draft tokens),
    some are admitted with a prompt's chunk, some are done, some give draft tokens back."""
    rng = random.Random(case["lens_seed"] + 7)
    old, new = [], []
    for n in _lens(case):
        u = rng.random()
        if case["tokens"] == 1 or u < 0.7:
            a, b = n, n + 1
        elif u < 0.8:
            a, b = 0, _logint(rng, 1, case["tokens"])
        elif u < 0.85:
            a, b = n, n + _logint(rng, 1, case["tokens"])
        elif u < 0.95:
            a, b = n, 0
        else:
            a, b = n, max(0, n - rng.randint(1, 8))
        old.append(a)
        new.append(b)
    return old, new


def _pages_of(n, page):
    return -(-n // page)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, gen, dt, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dt).mul_(std)


def _cache(case, n_pages, gen, dt):
    """Key and value caches [pages, page, heads, d] (views), filled."""
    _, hkv, d = HEADS[case["heads"]]
    page = case["page"]
    if case["layout"] == "joined":
        both = _normal((n_pages, 2, page, hkv, d), gen, dt)
        return both[:, 0], both[:, 1]
    if case["layout"] == "heads":
        return tuple(_normal((n_pages, hkv, page, d), gen, dt).transpose(1, 2) for _ in range(2))
    return tuple(_normal((n_pages, page, hkv, d), gen, dt) for _ in range(2))


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = _gen(seed)
    dt = torch.float32 if case["f32"] else torch.bfloat16
    hq, hkv, d = HEADS[case["heads"]]
    s = {"case": case}
    if case["kind"] == "pages":
        old, new = _page_lens(case)
        page = case["page"]
        width = max(_pages_of(max(a, b), page) for a, b in zip(old, new)) + 2
        held = [_pages_of(a, page) for a in old]
        n_pages = sum(held) + case["spare"]
        perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        col = torch.arange(width, device="cuda")
        have = torch.tensor(held, device="cuda")
        at = (torch.cumsum(have, 0) - have)[:, None] + col
        s["table"] = torch.where(col < have[:, None], perm[at.clamp(max=n_pages - 1)], 0).to(torch.int32)
        s["free_pages"] = torch.cat([perm[sum(held):], torch.zeros(sum(held), dtype=torch.int32, device="cuda")])
        s["free_in"] = _int32([case["spare"], 0])
        s["old_len"], s["new_len"] = _int32(old), _int32(new)
        n_new = sum(max(0, b - a) for a, b in zip(old, new))
        s["n_tok"] = -(-n_new // 64) * 64 + 64  # a captured batch's padding
        s["n_pages"] = n_pages
        s["free_out"] = torch.zeros_like(s["free_in"])
        s["seq_len"] = torch.zeros_like(s["old_len"])
        s["slots"] = torch.zeros(s["n_tok"], dtype=torch.int64, device="cuda")
        s["positions"] = torch.zeros(s["n_tok"], dtype=torch.int32, device="cuda")
        s["cu_new"] = torch.zeros(case["batch"] + 1, dtype=torch.int32, device="cuda")
        return s
    if case["kind"] in ("rope", "append"):
        n = case["tokens"]
        first = torch.randint(0, 100000, (1,), generator=gen, device="cuda")
        # long runs of tokens are prompts; a step's tokens sit anywhere
        pos = (first + torch.arange(n, device="cuda") % 8192 if n > 256 else
               torch.randint(0, 131072, (n,), generator=gen, device="cuda"))
        s["positions"] = pos.to(torch.int32)
        if case["kind"] == "rope":
            s["x"] = _normal((n, hq, d), gen, dt)
            s["out"] = torch.zeros_like(s["x"])
            return s
        s["qkv"] = _normal((n, (hq + 2 * hkv), d), gen, dt)  # the fused projection's rows
        n_pages = _pages_of(n + n // 8, case["page"]) + 2
        s["kcache"], s["vcache"] = _cache(case, n_pages, gen, dt)
        if n > 256:  # whole pages in any order, filled one token after the other
            p = torch.randperm(n_pages, generator=gen, device="cuda")
            i = torch.arange(n, device="cuda")
            s["slots"] = p[i // case["page"]] * case["page"] + i % case["page"]
        else:
            s["slots"] = torch.randperm(n_pages * case["page"], generator=gen, device="cuda")[:n]
            if n > 8:
                s["slots"][n // 2] = -1  # an idle slot of the batch
        s["q_out"] = torch.zeros((n, hq, d), dtype=dt, device="cuda")
        return s
    lens = _lens(case)
    page = case["page"]
    width = max(1, _pages_of(max(lens), page)) + 3
    n_pages = sum(_pages_of(n, page) for n in lens) + 5
    s["kcache"], s["vcache"] = _cache(case, n_pages, gen, dt)
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    have = torch.tensor([_pages_of(n, page) for n in lens], device="cuda")
    col = torch.arange(width, device="cuda")
    at = (torch.cumsum(have, 0) - have)[:, None] + col
    s["table"] = torch.where(col < have[:, None], perm[at.clamp(max=n_pages - 1)], -1).to(torch.int32)
    s["seq_len"] = _int32(lens)
    s["max_len"] = max(1, max(lens))
    s["q"] = _normal((case["batch"], hq, d), gen, dt, 2.0)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros((case["batch"], hq), dtype=torch.float32, device="cuda")
    return s


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _kept(s):
    """The descriptor, rotary table and workspace that a program makes once and keeps."""
    from paper_2607_24331_gb300 import dck
    case = s["case"]
    hq, _, d = HEADS[case["heads"]]
    k = {"dck": dck, "dtype": dck.DCK_F32 if case["f32"] else dck.DCK_BF16}
    if case["kind"] in ("rope", "append"):
        share, theta, layout, scaling, factor, a, b, trained, magnitude = ROPES[case["rope"]]
        k["rope"] = dck.Rope(int(d * share), theta, layout=layout, scaling=scaling, factor=factor, slow=a, fast=b,
                             trained_len=trained, magnitude=magnitude)
    if case["kind"] in ("append", "attend"):
        k["cache"] = dck.PagedCache.from_tensors(s["kcache"], s["vcache"], hq)
    if case["kind"] == "attend":
        k["ws_bytes"] = dck.dck_paged_decode_workspace_size(k["cache"], case["batch"], s["max_len"])
        k["ws"] = torch.empty(max(k["ws_bytes"], 256), dtype=torch.uint8, device="cuda")
    s["kept"] = k
    return k


def _run_own(s):
    k = s.get("kept") or _kept(s)
    dck, case = k["dck"], s["case"]
    kind = case["kind"]
    if kind == "pages":
        dck.check(dck.dck_page_update(case["batch"], case["page"], s["n_pages"], s["old_len"], s["new_len"], s["seq_len"],
                                      s["table"], s["table"].shape[1], s["free_pages"], s["free_in"], s["free_out"],
                                      s["n_tok"], s["slots"], s["positions"], s["cu_new"]), "dck_page_update")
        return {n: s[n] for n in ("table", "free_pages", "free_out", "seq_len", "slots", "positions", "cu_new")}
    hq, hkv, d = HEADS[case["heads"]]
    if kind == "rope":
        dck.check(dck.dck_rope(k["rope"], s["x"], case["tokens"], hq, d, k["dtype"], hq * d, d, s["positions"],
                               s["out"], hq * d, d, case["transpose"]), "dck_rope")
        return {"out": s["out"]}
    if kind == "append":
        row = (hq + 2 * hkv) * d
        q, kk, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
        dck.check(dck.dck_paged_append(k["cache"], k["rope"], q, row, kk, row, v, row, case["tokens"], s["positions"],
                                       s["slots"], s["q_out"], s["kcache"], s["vcache"]), "dck_paged_append")
        return {"q": s["q_out"], "kcache": s["kcache"], "vcache": s["vcache"]}
    dck.check(dck.dck_paged_decode_attention(k["cache"], s["q"], hq * d, s["kcache"], s["vcache"], s["table"],
                                             s["table"].shape[1], s["seq_len"], case["batch"], s["max_len"],
                                             1.0 / math.sqrt(d), case["window"], case["softcap"], s["out"], s["lse"],
                                             k["ws"], k["ws_bytes"]), "dck_paged_decode_attention")
    return {"out": s["out"], "lse": s["lse"]}


# --------------------------------------------------------------------------
# the plain form
# --------------------------------------------------------------------------

def _plain_pages(s):
    page = s["case"]["page"]
    old, new = s["old_len"].long(), s["new_len"].long()
    table, width = s["table"], s["table"].shape[1]
    f = s["free_in"][0].long()
    po, pn = (old + page - 1) // page, (new + page - 1) // page
    rel, grow = (po - pn).clamp(min=0), (pn - po).clamp(min=0)
    before = torch.cumsum(grow, 0) - grow
    n_rel = torch.cumsum(rel, 0)
    total = f + n_rel[-1]
    ok = (grow == 0) | (before + grow <= total)
    used = torch.where(ok & (grow > 0), before + grow, 0).max()
    left = total - used
    # every free page in order: the list, then the pages given back, by request and page
    col = torch.arange(width, device=table.device)
    back = (col >= pn[:, None]) & (col < po[:, None])
    pool = s["free_pages"].clone()
    j = torch.arange(pool.numel(), device=table.device)
    spot = torch.where(back, f + (n_rel - rel)[:, None] + col - pn[:, None], pool.numel())
    pool = torch.cat([pool, pool[:1]]).scatter(0, spot.reshape(-1), table.reshape(-1))[:-1]
    take = total - 1 - (before[:, None] + col - po[:, None])
    fresh = ok[:, None] & (col >= po[:, None]) & (col < pn[:, None])
    table = torch.where(fresh, pool[take.clamp(0, pool.numel() - 1)], table)
    free = torch.where((j >= f) & (j < left), pool, s["free_pages"])
    n_new = (new - old).clamp(min=0)
    cu = torch.cat([torch.zeros_like(n_new[:1]), torch.cumsum(n_new, 0)])
    i = torch.arange(s["n_tok"], device=table.device)
    b = (torch.searchsorted(cu, i, right=True) - 1).clamp(max=old.numel() - 1)
    live = i < cu[-1]
    pos = torch.where(live, old[b] + i - cu[b], 0)
    slot = table[b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    return {"table": table, "free_pages": free, "free_out": torch.stack([left, (~ok).sum()]).to(torch.int32),
            "seq_len": torch.where(ok, new, old).to(torch.int32), "slots": torch.where(live & ok[b], slot, -1),
            "positions": pos.to(torch.int32), "cu_new": cu.to(torch.int32)}


def _frequencies(rope, d):
    """The rotary frequencies (radians per position) as 64-bit fractions of a turn in signed integers."""
    share, theta, layout, scaling, factor, slow, fast, trained, magnitude = ROPES[rope]
    r = int(d * share)
    i = torch.arange(r // 2, dtype=torch.float64)
    if scaling == "ntk":
        theta = theta * factor ** (r / (r - 2))
    w = theta ** (-2.0 * i / r)
    if scaling == "linear":
        w = w / factor
    if scaling == "bands":
        mix = ((trained * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        w = (1 - mix) * w / factor + mix * w
    if scaling == "yarn":
        lo, hi = (r * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(theta)) for t in (fast, slow))
        lo, hi = max(0, math.floor(lo)), min(r - 1, math.ceil(hi))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = (1 - ramp) * w + ramp * w / factor
    return r, layout, magnitude, w


def _plain_rotate(x, pos, rope, transpose):
    r, layout, magnitude, w = _frequencies(rope, x.shape[-1])
    # angles in turns: position times a 64-bit fraction, whole turns falling off the top
    turns = w / (2 * math.pi)
    fraction = torch.round((turns - torch.floor(turns)) * 2.0 ** 62).to(torch.int64).to(x.device) << 2
    a = ((pos.long()[:, None] * fraction) >> 32).float() * (2 * math.pi / 2.0 ** 32)
    c, sn = (torch.cos(a) * magnitude)[:, None], (torch.sin(a) * magnitude)[:, None]
    sn = -sn if transpose else sn
    y = x.float()
    x1, x2 = (y[..., :r // 2], y[..., r // 2:r]) if layout == "half" else (y[..., 0:r:2], y[..., 1:r:2])
    z1, z2 = x1 * c - x2 * sn, x1 * sn + x2 * c
    z = torch.cat([z1, z2], -1) if layout == "half" else torch.stack([z1, z2], -1).flatten(-2)
    return torch.cat([z, y[..., r:]], -1).to(x.dtype)


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    page, lens = case["page"], s["seq_len"].long()
    t = torch.arange(s["max_len"], device=lens.device)
    live = t < lens[:, None]
    if case["window"]:
        live &= t >= lens[:, None] - case["window"]
    which = torch.where(live, s["table"][:, t // page].long(), 0)
    q = s["q"].float().view(case["batch"], hkv, hq // hkv, d) / math.sqrt(d)
    k = s["kcache"][which, t % page].float()
    x = torch.matmul(q, k.permute(0, 2, 3, 1))
    del k
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    dead = ~live[:, None, None]
    x = x.masked_fill(dead, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    v = s["vcache"][which, t % page].float().masked_fill(~live[:, :, None, None], 0.0)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)) / torch.where(total > 0, total, 1.0)
    return {"out": o.reshape(case["batch"], hq, d).to(s["q"].dtype),
            "lse": (m + torch.log(total)).reshape(case["batch"], hq)}


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "pages":
        return _plain_pages(s)
    hq, hkv, _ = HEADS[case["heads"]]
    if case["kind"] == "rope":
        return {"out": _plain_rotate(s["x"], s["positions"], case["rope"], case["transpose"])}
    if case["kind"] == "append":
        q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
        slots = s["slots"]
        keep = slots >= 0
        at, off = slots[keep] // case["page"], slots[keep] % case["page"]
        s["kcache"][at, off] = _plain_rotate(k, s["positions"], case["rope"], False)[keep]
        s["vcache"][at, off] = v[keep]
        return {"q": _plain_rotate(q, s["positions"], case["rope"], False), "kcache": s["kcache"], "vcache": s["vcache"]}
    return _plain_attend(s)


def run(s):
    return _run_own(s) if own else _run_plain(s)


# --------------------------------------------------------------------------
# work and the definition in 64 bits
# --------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once; the products of scores and values, the rotations."""
    hq, hkv, d = HEADS[case["heads"]]
    el = 4 if case["f32"] else 2
    if case["kind"] == "pages":
        old, new = _page_lens(case)
        page = case["page"]
        moved = sum(abs(_pages_of(a, page) - _pages_of(b, page)) for a, b in zip(old, new))
        n_new = sum(max(0, b - a) for a, b in zip(old, new))
        return {"bytes": 16 * len(old) + 8 * moved + 12 * n_new, "flops": 0}
    n = case["tokens"]
    if case["kind"] == "rope":
        return {"bytes": 2 * el * n * hq * d + 4 * n, "flops": 3 * n * hq * d}
    if case["kind"] == "append":
        return {"bytes": 2 * el * n * (hq + 2 * hkv) * d + 12 * n, "flops": 3 * n * (hq + hkv) * d}
    rows = sum(min(x, case["window"] or x) for x in _lens(case))
    return {"bytes": el * (2 * rows * hkv * d + 2 * case["batch"] * hq * d) + 4 * rows // case["page"] + 4 * case["batch"] * (hq + 1),
            "flops": 4 * rows * hq * d}


def _exact_rotate(x, pos, rope, transpose):
    r, layout, magnitude, w = _frequencies(rope, x.shape[-1])
    e = torch.polar(torch.full_like(pos, magnitude, dtype=torch.float64)[:, None].expand(-1, r // 2),
                    pos.double()[:, None] * w.to(x.device))[:, None]
    e = e.conj() if transpose else e
    y = x.double().clone()
    if layout == "half":
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * e
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :r].reshape(*y.shape[:-1], r // 2, 2)) * e
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, d = HEADS[case["heads"]]
    if case["kind"] == "pages":
        return None  # whole numbers
    if case["kind"] == "rope":
        return {"out": _exact_rotate(s["x"], s["positions"], case["rope"], case["transpose"])}
    page = case["page"]
    if case["kind"] == "append":
        kc, vc = s["kcache"].double(), s["vcache"].double()
        k = _exact_rotate(s["qkv"][:, hq:hq + hkv], s["positions"], case["rope"], False)
        keep = torch.nonzero(s["slots"] >= 0).squeeze(1)
        at = s["slots"][keep]
        kc[at // page, at % page] = k[keep]
        vc[at // page, at % page] = s["qkv"][keep, hq + hkv:].double()
        return {"q": _exact_rotate(s["qkv"][:, :hq], s["positions"], case["rope"], False), "kcache": kc, "vcache": vc}
    g = hq // hkv
    out = torch.zeros((case["batch"], hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], hq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(case)):
        if n == 0:
            continue
        first = max(0, n - case["window"]) if case["window"] else 0
        t = torch.arange(first, n, device="cuda")
        rows = s["table"][b, t // page].long(), t % page
        for h in range(hkv):
            k, v = (c[rows[0], rows[1], h].double() for c in (s["kcache"], s["vcache"]))
            x = s["q"][b, h * g:(h + 1) * g].double() @ k.T / math.sqrt(d)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            out[b, h * g:(h + 1) * g] = torch.softmax(x, -1) @ v
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(x, -1)
    return {"out": out, "lse": lse}
