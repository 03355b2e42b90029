"""An 8-bit paged key-value cache and attention over shared prefixes, as cases to be timed and compared.

Every case is one call of a public entry point of ``dck``, or the same in elementary torch operations.  Kinds:

  append  dck_quant_append: new tokens' queries rotated, keys rotated, both keys and values
          rounded to 8 bits with a scale for each token and head and written to their rows
  read    dck_quant_read: rows of the cache as the values they stand for
  attend  dck_quant_decode_attention: one query per sequence over 8-bit pages
  shared  dck_paged_shared_attention (16-bit pages) or dck_quant_shared_attention (8-bit pages):
          one query per row, where the rows of a group begin with the same tokens, in the same pages

A row of 8 bits: s = 2^e, e the smallest whole number (-126 at least) for which the largest magnitude is at
most 448 s; codes are e4m3 of x / s.  What is quantised has the type of the new tokens: a rotated key is rounded to it first.

Lengths are ``lo == hi`` (all alike) or ragged, drawn log-uniformly from [lo, hi] with ``lens_seed``; ``idle`` of the
sequences are empty (the padding of a captured batch).  For ``shared`` they are what a group shares, ``own`` what each row
has after it: ``users`` rows of a group are requests that begin with one prompt (whole pages) and go on by up to ``own``
tokens, or, with ``chunk``, the new tokens of one request, each seeing those before it.
Cache ``layout``: "rows" [pages, page, heads, d], keys and values apart; "joined" one buffer [pages, 2, page, heads, d];
"heads" [pages, heads, page, d].
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
    "bands": (1.0, 5e5, "half", "bands", 8.0, 1.0, 4.0, 8192, 1.0),
    "part": (0.5, 1e4, "interleaved", "none", 1.0, 0.0, 0.0, 0, 1.0),
}


def _case(name, kind, **kw):
    c = dict(kind=kind, heads="gqa8", f32=False, q8=True, batch=1, lo=1, hi=1, idle=0, page=16, layout="rows", window=0,
             softcap=0.0, tokens=0, rope="plain", users=0, own=0, chunk=False, lens_seed=1)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the new tokens of one step of a few users: latency
        _case("append-b8", "append", tokens=8, rope="bands"),
        # a long prompt pair of 2 x 8192 tokens, into a joined cache
        _case("append-16384", "append", tokens=16384, page=64, rope="bands", layout="joined"),
        # one conversation's keys and values of a small fp32 layer back in full width
        _case("read-f32-777", "read", heads="mha8", f32=True, tokens=777, page=24),
        # two long documents' prefixes back in full width, for a prompt's attention
        _case("read-65536", "read", tokens=65536, page=64),
        # one user in a short conversation: latency
        _case("attend-gqa-b1-777", "attend", batch=1, lo=777, hi=777),
        # a few users of a layer with a head dim that is no power of two, queries and outputs in fp32
        _case("attend-f32-odd-b4", "attend", heads="odd", f32=True, batch=4, lo=300, hi=2000, page=24),
        # the ordinary serving batch on the 32-head layer
        _case("attend-mha-b16-4096", "attend", heads="mha32", batch=16, lo=4096, hi=4096, page=32),
        # a continuous batch, every sequence of another length, some slots idle
        _case("attend-gqa-b32-ragged", "attend", batch=32, lo=1024, hi=32768, idle=3, layout="joined"),
        # four users who begin with one short prompt, 16-bit cache: latency
        _case("shared-gqa-b4-512", "shared", q8=False, batch=1, users=4, lo=512, hi=512, own=64),
        # an assistant's long instructions and 64 users' conversations, 16-bit cache
        _case("shared-gqa-b64-8192", "shared", q8=False, batch=1, users=64, lo=8192, hi=8192, own=1024, page=32),
        # chunks of 32 tokens of four long prompts, 16-bit cache
        _case("shared-chunk-4x32", "shared", q8=False, batch=4, users=32, lo=4000, hi=9000, chunk=True),
        # 16 questions on one long document, 8-bit cache of the 32-head layer
        _case("shared-q8-mha-b16-32768", "shared", heads="mha32", batch=1, users=16, lo=32768, hi=32768, own=256, page=64),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MAX_ATTEND = 2 * 131072 * 8 * 128    # key elements of an attend call, padded to its longest sequence
MAX_SHARED = 16 * 32768 * 32 * 128   # key elements that the rows of a shared call see


def draw(rng):
    kind = rng.choice(("append", "read", "attend", "attend", "shared", "shared"))
    seed = rng.randrange(1 << 20)
    page = rng.choice((1, 8, 16, 16, 24, 32, 64, 100, 128, 256))
    layout = rng.choice(("rows", "joined", "heads"))
    f32 = rng.random() < 0.2
    heads = rng.choice(("mha32", "gqa8", "gqa8", "mha8", "mqa", "odd", "wide"))
    hq, hkv, d = HEADS[heads]
    if kind in ("append", "read"):
        most = 16384 * 48 * 128 // ((hq + 2 * hkv) * d) if kind == "append" else 65536 * 8 * 128 // (hkv * d)
        return _case(None, kind, heads=heads, f32=f32, tokens=_logint(rng, 1, most // (2 if f32 else 1)), page=page,
                     layout=layout, rope=rng.choice(sorted(ROPES)), lens_seed=seed)
    window, softcap = rng.choice((0, 0, 0, _logint(rng, 1, 4096))), rng.choice((0.0, 0.0, 30.0))
    if kind == "attend":
        while True:
            batch, hi = _logint(rng, 1, 128), _logint(rng, 1, 131072)
            if batch * hi * hkv * d <= MAX_ATTEND:
                break
        return _case(None, kind, heads=heads, f32=f32, batch=batch, lo=rng.choice((hi, max(1, hi // 16))), hi=hi,
                     idle=rng.choice((0, 0, batch // 8)), page=page, layout=layout, window=window, softcap=softcap,
                     lens_seed=seed)
    chunk = rng.random() < 0.4
    while True:
        batch, users, hi, more = _logint(rng, 1, 16), _logint(rng, 1, 128), _logint(rng, 1, 32768), _logint(rng, 1, 2048)
        if chunk:
            more = 0
        if batch * users * (hi + more + 256) * hkv * d <= MAX_SHARED:
            break
    return _case(None, kind, heads=heads, f32=f32, q8=rng.random() < 0.5, batch=batch, users=users,
                 lo=rng.choice((hi, max(1, hi // 16))), hi=hi, own=more, chunk=chunk, idle=rng.choice((0, 0, batch * users // 8)),
                 page=page, layout=layout, window=window, softcap=softcap, lens_seed=seed)


def _lens(case):
    rng = random.Random(case["lens_seed"])
    lens = [_logint(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    if case["kind"] == "shared":
        return lens
    for b in rng.sample(range(case["batch"]), case["idle"]):
        lens[b] = 0
    return lens


def _shared(case):
    """(tokens that each group shares, lengths of all rows, groups one after the other)."""
    rng = random.Random(case["lens_seed"] + 3)
    share, rows = [], []
    for n in _lens(case):
        if case["chunk"]:  # the last of n tokens and its predecessors
            first = max(0, n - case["users"])
            share.append(first + case["users"])
            rows += [first + 1 + i for i in range(case["users"])]
        else:
            share.append(_pages_of(n, case["page"]) * case["page"])
            rows += [share[-1] + _logint(rng, 1, case["own"]) for _ in range(case["users"])]
    for b in rng.sample(range(len(rows)), case["idle"]):
        rows[b] = 0
    return share, rows


def _pages_of(n, page):
    return -(-n // page)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, gen, dt, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dt).mul_(std)


def _views(make, shape, layout):
    """Two [pages, page, heads, ...] views of one or two buffers."""
    n_pages, page, hkv = shape[:3]
    if layout == "joined":
        both = make((n_pages, 2, page, hkv) + shape[3:])
        return both[:, 0], both[:, 1]
    if layout == "heads":
        return tuple(make((n_pages, hkv, page) + shape[3:]).transpose(1, 2) for _ in range(2))
    return tuple(make(shape) for _ in range(2))


def _codes(shape, gen):
    """8-bit rows as appends leave them: magnitudes up to 448, a sixth to a third of that as a rule."""
    return _normal(shape, gen, torch.bfloat16, 120.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _scales(shape, gen):
    return torch.exp2(torch.randint(-8, -5, shape, generator=gen, device="cuda").float())


def _caches(s, n_pages, gen, dt):
    """Key and value caches, filled, with the scales of 8-bit ones."""
    case = s["case"]
    _, hkv, d = HEADS[case["heads"]]
    shape = (n_pages, case["page"], hkv)
    if case["q8"]:
        s["kcache"], s["vcache"] = _views(lambda x: _codes(x, gen), shape + (d,), case["layout"])
        s["k_scale"], s["v_scale"] = _views(lambda x: _scales(x, gen), shape, case["layout"])
    else:
        s["kcache"], s["vcache"] = _views(lambda x: _normal(x, gen, dt), shape + (d,), case["layout"])


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _slots(n, case, n_pages, gen):
    """Rows of n tokens: whole pages in any order for long runs, else rows anywhere."""
    if n > 256:
        p = torch.randperm(n_pages, generator=gen, device="cuda")
        i = torch.arange(n, device="cuda")
        return p[i // case["page"]] * case["page"] + i % case["page"]
    return torch.randperm(n_pages * case["page"], generator=gen, device="cuda")[:n]


def prepare(case, seed):
    gen = _gen(seed)
    dt = torch.float32 if case["f32"] else torch.bfloat16
    hq, hkv, d = HEADS[case["heads"]]
    page = case["page"]
    s = {"case": case}
    if case["kind"] in ("append", "read"):
        n = case["tokens"]
        n_pages = _pages_of(n + n // 8, page) + 2
        _caches(s, n_pages, gen, dt)
        s["slots"] = _slots(n, case, n_pages, gen)
        if n > 8:
            s["slots"][n // 2] = -1  # an idle slot of the batch
        if case["kind"] == "read":
            s["k"], s["v"] = (torch.zeros((n, hkv, d), dtype=dt, device="cuda") for _ in range(2))
            return s
        first = torch.randint(0, 100000, (1,), generator=gen, device="cuda")
        # long runs of tokens are prompts; a step's tokens sit anywhere
        pos = (first + torch.arange(n, device="cuda") % 8192 if n > 256 else
               torch.randint(0, 131072, (n,), generator=gen, device="cuda"))
        s["positions"] = pos.to(torch.int32)
        s["qkv"] = _normal((n, (hq + 2 * hkv), d), gen, dt)  # the fused projection's rows
        s["q_out"] = torch.zeros((n, hq, d), dtype=dt, device="cuda")
        return s
    # tables: `held` pages of each row; a group's rows begin with its shared pages
    if case["kind"] == "shared":
        share, lens = _shared(case)
        users = case["users"]
        whole = torch.tensor([_pages_of(n, page) for n in share], device="cuda").repeat_interleave(users)
        s["shared_len"] = _int32(share)
        s["group_start"] = _int32([g * users for g in range(case["batch"] + 1)])
        group = torch.arange(len(lens), device="cuda") // users
        mine = (torch.tensor([_pages_of(n, page) for n in lens], device="cuda") - whole).clamp(min=0)
        # groups of one row share nothing: all of it is their own
        s["max_own"] = max([1] + [n - (share[b // users] if users > 1 else 0) for b, n in enumerate(lens)])
    else:
        lens = _lens(case)
        whole = torch.zeros(len(lens), dtype=torch.int64, device="cuda")
        group = torch.arange(len(lens), device="cuda")
        mine = torch.tensor([_pages_of(n, page) for n in lens], device="cuda")
        users = 1
    held = whole + mine
    width = int(held.max()) + 3
    n_groups = len(lens) // users
    shared_pages = int(whole.view(n_groups, users)[:, 0].sum())
    n_pages = shared_pages + int(mine.sum()) + 5
    _caches(s, n_pages, gen, dt)
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(width, device="cuda")
    per_group = whole.view(n_groups, users)[:, 0]
    at_group = (torch.cumsum(per_group, 0) - per_group)[group][:, None] + col
    at_mine = shared_pages + (torch.cumsum(mine, 0) - mine)[:, None] + col - whole[:, None]
    at = torch.where(col < whole[:, None], at_group, at_mine).clamp(0, n_pages - 1)
    s["table"] = torch.where(col < held[:, None], perm[at], -1).to(torch.int32)
    s["seq_len"] = _int32(lens)
    s["max_len"] = max(1, max(lens))
    s["q"] = _normal((len(lens), hq, d), gen, dt, 2.0)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros((len(lens), hq), dtype=torch.float32, device="cuda")
    return s


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _kept(s):
    """The descriptor, rotary table and workspace that a program makes once and keeps."""
    from paper_2607_24331_gb300 import dck
    case = s["case"]
    hq, _, d = HEADS[case["heads"]]
    k = {"dck": dck}
    if case["kind"] == "append":
        share, theta, layout, scaling, factor, a, b, trained, magnitude = ROPES[case["rope"]]
        k["rope"] = dck.Rope(int(d * share), theta, layout=layout, scaling=scaling, factor=factor, slow=a, fast=b,
                             trained_len=trained, magnitude=magnitude)
    if case["q8"]:
        k["cache"] = dck.QuantCache.from_tensors(s["kcache"], s["k_scale"], s["vcache"], s["v_scale"], hq,
                                                 "f32" if case["f32"] else "bf16")
    else:
        k["cache"] = dck.PagedCache.from_tensors(s["kcache"], s["vcache"], hq)
    n = s["seq_len"].numel() if "seq_len" in s else 0
    if case["kind"] == "attend":
        k["ws_bytes"] = dck.dck_quant_decode_workspace_size(k["cache"], n, s["max_len"])
    if case["kind"] == "shared":
        size = dck.dck_quant_shared_workspace_size if case["q8"] else dck.dck_paged_shared_workspace_size
        k["ws_bytes"] = size(k["cache"], n, s["max_len"], s["max_own"])
    if "ws_bytes" in k:
        k["ws"] = torch.empty(max(k["ws_bytes"], 256), dtype=torch.uint8, device="cuda")
    s["kept"] = k
    return k


def _run_own(s):
    k = s.get("kept") or _kept(s)
    dck, case = k["dck"], s["case"]
    kind = case["kind"]
    hq, hkv, d = HEADS[case["heads"]]
    if kind == "append":
        row = (hq + 2 * hkv) * d
        q, kk, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
        dck.check(dck.dck_quant_append(k["cache"], k["rope"], q, row, kk, row, v, row, case["tokens"], s["positions"],
                                       s["slots"], s["q_out"], s["kcache"], s["k_scale"], s["vcache"], s["v_scale"]),
                  "dck_quant_append")
        return _written(s, s["q_out"])
    if kind == "read":
        dck.check(dck.dck_quant_read(k["cache"], case["tokens"], s["slots"], s["kcache"], s["k_scale"], s["vcache"],
                                     s["v_scale"], s["k"], hkv * d, s["v"], hkv * d), "dck_quant_read")
        return {"k": s["k"], "v": s["v"]}
    n = s["seq_len"].numel()
    if kind == "attend":
        dck.check(dck.dck_quant_decode_attention(k["cache"], s["q"], hq * d, s["kcache"], s["k_scale"], s["vcache"],
                                                 s["v_scale"], s["table"], s["table"].shape[1], s["seq_len"], n,
                                                 s["max_len"], 1.0 / math.sqrt(d), case["window"], case["softcap"],
                                                 s["out"], s["lse"], k["ws"], k["ws_bytes"]), "dck_quant_decode_attention")
        return {"out": s["out"], "lse": s["lse"]}
    if case["q8"]:
        dck.check(dck.dck_quant_shared_attention(k["cache"], s["q"], hq * d, s["kcache"], s["k_scale"], s["vcache"],
                                                 s["v_scale"], s["table"], s["table"].shape[1], s["seq_len"], n,
                                                 s["max_len"], s["max_own"], case["batch"], s["group_start"],
                                                 s["shared_len"], 1.0 / math.sqrt(d), case["window"], case["softcap"],
                                                 s["out"], s["lse"], k["ws"], k["ws_bytes"]), "dck_quant_shared_attention")
    else:
        dck.check(dck.dck_paged_shared_attention(k["cache"], s["q"], hq * d, s["kcache"], s["vcache"], s["table"],
                                                 s["table"].shape[1], s["seq_len"], n, s["max_len"], s["max_own"],
                                                 case["batch"], s["group_start"], s["shared_len"], 1.0 / math.sqrt(d),
                                                 case["window"], case["softcap"], s["out"], s["lse"], k["ws"],
                                                 k["ws_bytes"]), "dck_paged_shared_attention")
    return {"out": s["out"], "lse": s["lse"]}


def _written(s, q):
    e4m3 = torch.float8_e4m3fn
    return {"q": q, "kcache": s["kcache"].view(e4m3), "k_scale": s["k_scale"], "vcache": s["vcache"].view(e4m3),
            "v_scale": s["v_scale"]}


# --------------------------------------------------------------------------
# the plain form
# --------------------------------------------------------------------------

def _frequencies(rope, d):
    """The rotary frequencies (radians per position), in 64 bits."""
    share, theta, layout, scaling, factor, slow, fast, trained, magnitude = ROPES[rope]
    r = int(d * share)
    i = torch.arange(r // 2, dtype=torch.float64)
    w = theta ** (-2.0 * i / r)
    if scaling == "linear":
        w = w / factor
    if scaling == "bands":
        mix = ((trained * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        w = (1 - mix) * w / factor + mix * w
    return r, layout, magnitude, w


def _plain_rotate(x, pos, rope):
    r, layout, magnitude, w = _frequencies(rope, x.shape[-1])
    # angles in turns: position times a 64-bit fraction, whole turns falling off the top
    turns = w / (2 * math.pi)
    fraction = torch.round((turns - torch.floor(turns)) * 2.0 ** 62).to(torch.int64).to(x.device) << 2
    a = ((pos.long()[:, None] * fraction) >> 32).float() * (2 * math.pi / 2.0 ** 32)
    c, sn = (torch.cos(a) * magnitude)[:, None], (torch.sin(a) * magnitude)[:, None]
    y = x.float()
    x1, x2 = (y[..., :r // 2], y[..., r // 2:r]) if layout == "half" else (y[..., 0:r:2], y[..., 1:r:2])
    z1, z2 = x1 * c - x2 * sn, x1 * sn + x2 * c
    z = torch.cat([z1, z2], -1) if layout == "half" else torch.stack([z1, z2], -1).flatten(-2)
    return torch.cat([z, y[..., r:]], -1).to(x.dtype)


def _plain_quantise(x):
    """(codes, scales) of rows: powers of two, so that the quotients are exact."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))  # m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    e = (e - 9 + (m > 0.875)).clamp(min=-126)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), torch.ldexp(torch.ones_like(m), e)


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d = HEADS[case["heads"]]
    page, lens = case["page"], s["seq_len"].long()
    n = lens.numel()
    t = torch.arange(s["max_len"], device=lens.device)
    live = t < lens[:, None]
    if case["window"]:
        live &= t >= lens[:, None] - case["window"]
    which = torch.where(live, s["table"][:, t // page].long(), 0)
    values = lambda c, f: (s[c].view(torch.float8_e4m3fn)[which, t % page].float() * s[f][which, t % page][..., None]  # noqa: E731
                           if case["q8"] else s[c][which, t % page].float())
    q = s["q"].float().view(n, hkv, hq // hkv, d) / math.sqrt(d)
    k = values("kcache", "k_scale")
    x = torch.matmul(q, k.permute(0, 2, 3, 1))
    del k
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    x = x.masked_fill(~live[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    v = values("vcache", "v_scale").masked_fill(~live[:, :, None, None], 0.0)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)) / torch.where(total > 0, total, 1.0)
    return {"out": o.reshape(n, hq, d).to(s["q"].dtype), "lse": (m + torch.log(total)).reshape(n, hq)}


def _run_plain(s):
    case = s["case"]
    hq, hkv, _ = HEADS[case["heads"]]
    if case["kind"] in ("attend", "shared"):
        return _plain_attend(s)
    page, slots = case["page"], s["slots"]
    keep = slots >= 0
    if case["kind"] == "read":
        at, off = slots.clamp(min=0) // page, slots.clamp(min=0) % page
        for name, c, f in (("k", "kcache", "k_scale"), ("v", "vcache", "v_scale")):
            x = s[c].view(torch.float8_e4m3fn)[at, off].float() * s[f][at, off][..., None]
            s[name].copy_(torch.where(keep[:, None, None], x, 0.0))
        return {"k": s["k"], "v": s["v"]}
    at, off = slots[keep] // page, slots[keep] % page
    k = _plain_rotate(s["qkv"][:, hq:hq + hkv], s["positions"], case["rope"])
    for x, c, f in ((k, "kcache", "k_scale"), (s["qkv"][:, hq + hkv:], "vcache", "v_scale")):
        s[c][at, off], s[f][at, off] = _plain_quantise(x[keep])
    return _written(s, _plain_rotate(s["qkv"][:, :hq], s["positions"], case["rope"]))


def run(s):
    return _run_own(s) if own else _run_plain(s)


# --------------------------------------------------------------------------
# work and the definition in 64 bits
# --------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once; the products of scores and values, the rotations."""
    hq, hkv, d = HEADS[case["heads"]]
    el = 4 if case["f32"] else 2
    row = hkv * (d + 4 if case["q8"] else d * el)  # a token's keys, or values
    n = case["tokens"]
    if case["kind"] == "append":
        return {"bytes": el * n * (2 * hq + 2 * hkv) * d + 2 * n * row + 12 * n, "flops": n * (3 * hq + 7 * hkv) * d}
    if case["kind"] == "read":
        return {"bytes": 2 * n * row + 2 * el * n * hkv * d + 8 * n, "flops": 2 * n * hkv * d}
    seen = lambda x: min(x, case["window"] or x)  # noqa: E731
    if case["kind"] == "attend":
        lens = _lens(case)
        rows = tokens = sum(map(seen, lens))
    else:
        share, lens = _shared(case)
        rows, tokens, u = sum(map(seen, lens)), 0, case["users"]
        for g, p in enumerate(share):
            mine = lens[g * u:(g + 1) * u]
            first = min((max(0, x - seen(x)) for x in mine if x), default=p)
            tokens += max(0, min(p, max(mine)) - first) + sum(x - max(p, x - seen(x)) for x in mine if x > p)
    n = len(lens)
    return {"bytes": 2 * tokens * row + 2 * el * n * hq * d + 4 * tokens // case["page"] + 4 * n * (hq + 1),
            "flops": 4 * rows * hq * d}


def _exact_rotate(x, pos, rope):
    r, layout, magnitude, w = _frequencies(rope, x.shape[-1])
    e = torch.polar(torch.full_like(pos, magnitude, dtype=torch.float64)[:, None].expand(-1, r // 2),
                    pos.double()[:, None] * w.to(x.device))[:, None]
    y = x.double().clone()
    if layout == "half":
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * e
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :r].reshape(*y.shape[:-1], r // 2, 2)) * e
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_quantise(x):
    """(values of the codes, scales): the nearest multiple of the spacing at each magnitude, ties to even."""
    top = x.abs().amax(-1)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)  # the logarithm's own rounding
    e = torch.where(448.0 * torch.exp2(e) < top, e + 1, e).clamp(min=-126)
    y = x / torch.exp2(e)[..., None]
    spacing = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / spacing) * spacing, torch.exp2(e)


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, d = HEADS[case["heads"]]
    page = case["page"]
    e4m3 = torch.float8_e4m3fn
    if case["kind"] in ("append", "read"):
        keep = torch.nonzero(s["slots"] >= 0).squeeze(1)
        at, off = s["slots"][keep] // page, s["slots"][keep] % page
        if case["kind"] == "read":
            k, v = (torch.zeros((case["tokens"], hkv, d), dtype=torch.float64, device="cuda") for _ in range(2))
            for x, c, f in ((k, "kcache", "k_scale"), (v, "vcache", "v_scale")):
                x[keep] = s[c].view(e4m3)[at, off].double() * s[f][at, off].double()[..., None]
            return {"k": k, "v": v}
        found = {"q": _exact_rotate(s["qkv"][:, :hq], s["positions"], case["rope"])}
        key = _exact_rotate(s["qkv"][:, hq:hq + hkv], s["positions"], case["rope"])
        key = key.to(s["qkv"].dtype).double()  # rounded to the tokens' type first
        for x, c, f in ((key, "kcache", "k_scale"), (s["qkv"][:, hq + hkv:].double(), "vcache", "v_scale")):
            found[c], found[f] = s[c].view(e4m3).double(), s[f].double()
            found[c][at, off], found[f][at, off] = _exact_quantise(x[keep])
        return found
    g, lens = hq // hkv, s["seq_len"].tolist()
    out = torch.zeros((len(lens), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((len(lens), hq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n == 0:
            continue
        first = max(0, n - case["window"]) if case["window"] else 0
        t = torch.arange(first, n, device="cuda")
        p, o = s["table"][b, t // page].long(), t % page
        for h in range(hkv):
            if case["q8"]:
                k, v = (s[c].view(e4m3)[p, o, h].double() * s[f][p, o, h].double()[:, None]
                        for c, f in (("kcache", "k_scale"), ("vcache", "v_scale")))
            else:
                k, v = (s[c][p, o, h].double() for c in ("kcache", "vcache"))
            x = s["q"][b, h * g:(h + 1) * g].double() @ k.T / math.sqrt(d)
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            out[b, h * g:(h + 1) * g] = torch.softmax(x, -1) @ v
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(x, -1)
    return {"out": out, "lse": lse}
