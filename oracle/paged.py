"""Plain definitions for uncompressed layers over a paged cache (fp64 numpy, test infrastructure only).

Page bookkeeping is a sequential program on lists; rotations are complex
multiplications; attention loops over sequences and heads.
"""

import math

import numpy as np


def page_update(page_size, old_len, new_len, block_table, free_pages, n_free, n_tok, n_pages=None):
    """One step's bookkeeping, request by request, on lists.  With n_pages, page numbers outside [0, n_pages) refuse:
    one in the partly filled last page of a request that grows refuses that request alone; one among the pages that
    would be taken ends the list, so that its request and the later ones that ask for pages are refused.

    Returns a dict with block_table, free_pages, free (left, refused), seq_len, slots, positions, cu_new."""
    table = np.array(block_table, dtype=np.int64)
    pool = [int(p) for p in free_pages[:n_free]]
    pages = lambda n: -(-int(n) // page_size)  # noqa: E731
    outside = lambda p: n_pages is not None and not 0 <= p < n_pages  # noqa: E731
    broken = [n > o and o % page_size and outside(table[b, int(o) // page_size])
              for b, (o, n) in enumerate(zip(old_len, new_len))]
    for b, (o, n) in enumerate(zip(old_len, new_len)):
        pool += [int(table[b, c]) for c in range(pages(n), pages(o))]
    total = limit = len(pool)
    asked = refused = tokens = 0
    granted, seq_len = [], []
    for b, (o, n) in enumerate(zip(old_len, new_len)):
        want = 0 if broken[b] else max(0, pages(n) - pages(o))
        asked += want
        tokens += max(0, int(n) - int(o))
        late = n > o and tokens > n_tok  # no room for its slots
        if want and not late and asked <= limit:
            for x in range(asked - want, asked):  # the x-th page from the list's end
                if outside(pool[total - 1 - x]):
                    limit = x
                    break
        short = want > 0 and asked > limit
        refused += short
        granted.append(not (broken[b] or late or short))
        seq_len.append(int(n) if granted[b] else int(o))
        if granted[b]:
            for c in range(pages(o), pages(o) + want):
                table[b, c] = pool.pop()
    slots, positions, cu = [], [], [0]
    for b, (o, n) in enumerate(zip(old_len, new_len)):
        for t in range(int(o), int(n)):
            positions.append(t)
            slots.append(int(table[b, t // page_size]) * page_size + t % page_size if granted[b] else -1)
        cu.append(len(positions))
    pad = n_tok - len(slots)
    free = np.array(free_pages, dtype=np.int64)
    free[n_free:max(n_free, len(pool))] = pool[n_free:]
    return dict(block_table=table, free_pages=free, free=np.array([len(pool), refused]), seq_len=np.array(seq_len),
                slots=np.array((slots + [-1] * pad)[:n_tok]), positions=np.array((positions + [0] * pad)[:n_tok]),
                cu_new=np.array(cu))


def rope_frequencies(rotary_dim, theta, scaling="none", factor=1.0, slow=1.0, fast=32.0, trained_len=0):
    """Radians per position of each pair."""
    out = []
    for i in range(rotary_dim // 2):
        base = theta * factor ** (rotary_dim / (rotary_dim - 2)) if scaling == "ntk" else theta
        w = base ** (-2.0 * i / rotary_dim)
        if scaling == "linear":
            w /= factor
        elif scaling == "bands":
            turns = trained_len * w / (2 * math.pi)
            mix = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
            w = (1 - mix) * w / factor + mix * w
        elif scaling == "yarn":
            pair = lambda n: rotary_dim * math.log(trained_len / (2 * math.pi * n)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(0, math.floor(pair(fast))), min(rotary_dim - 1, math.ceil(pair(slow)))
            ramp = min(1.0, max(0.0, (i - a) / max(b - a, 1e-3)))
            w = (1 - ramp) * w + ramp * w / factor
        out.append(w)
    return np.array(out)


def rotate(x, positions, frequencies, layout="half", magnitude=1.0, transpose=False):
    """x [n_tok, heads, d] rotated at positions [n_tok]; the transpose turns back."""
    x = np.asarray(x, dtype=np.float64)
    r = 2 * len(frequencies)
    turn = magnitude * np.exp((-1j if transpose else 1j) * np.outer(positions, frequencies))[:, None, :]
    y = x.copy()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = (x[..., first] + 1j * x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def paged_decode(q, kcache, vcache, block_table, seq_len, scale, window=0, softcap=0.0):
    """(out [B, Hq, d], lse [B, Hq], weight [B, Hq, d], slack [B, Hq]) over caches [pages, page, Hkv, d]:
    weight = sum_t p_t |v_t| and slack = max_t scale * sum |q| |k_t|, the quantities that rounding errors scale with."""
    B, hq, d = q.shape
    page, hkv = kcache.shape[1], kcache.shape[2]
    out, weight = np.zeros((B, hq, d)), np.zeros((B, hq, d))
    lse, slack = np.full((B, hq), -np.inf), np.zeros((B, hq))
    for b in range(B):
        n = int(seq_len[b])
        t = np.arange(max(0, n - window) if window else 0, n)
        if not len(t):
            continue
        p, o = np.asarray(block_table)[b, t // page], t % page
        for h in range(hkv):
            k, v = kcache[p, o, h].astype(np.float64), vcache[p, o, h].astype(np.float64)
            for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                s = scale * (k @ q[b, j])
                if softcap:
                    s = softcap * np.tanh(s / softcap)
                m = s.max()
                e = np.exp(s - m)
                out[b, j] = e @ v / e.sum()
                weight[b, j] = e @ np.abs(v) / e.sum()
                lse[b, j] = m + math.log(e.sum())
                slack[b, j] = abs(scale) * (np.abs(k) @ np.abs(q[b, j])).max()
    return out, lse, weight, slack
