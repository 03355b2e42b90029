"""The paged cache's entry points refuse what they cannot take, before any CUDA call (fake aligned addresses, never
dereferenced), and dck_rope_init's frequencies are the formulas'."""

import math

import numpy as np
import pytest

from oracle import paged as P
from paper_2607_24331_gb300 import dck
from paged_util import ROPES

A = 1 << 20  # an aligned address that nothing reads
INVALID, UNSUPPORTED = dck.DCK_ERR_INVALID, dck.DCK_ERR_UNSUPPORTED


def _cache(**kw):
    a = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, dtype="bf16")
    a.update(kw)
    return dck.PagedCache(**a)


@pytest.mark.parametrize("kw,expect", [
    (dict(), dck.DCK_OK), (dict(n_q_heads=8, n_kv_heads=8, head_dim=8, page_size=1, n_pages=1), dck.DCK_OK),
    (dict(n_q_heads=128, n_kv_heads=1, head_dim=256, page_size=65536, dtype="f32"), dck.DCK_OK),
    (dict(n_q_heads=30), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_heads=-1), INVALID), (dict(head_dim=0), INVALID),
    (dict(page_size=0), INVALID), (dict(n_pages=0), INVALID), (dict(head_dim=100), UNSUPPORTED),
    (dict(head_dim=264), UNSUPPORTED), (dict(page_size=65537), UNSUPPORTED),
    (dict(k_strides=(16384, 1024, 0)), INVALID), (dict(v_strides=(16384, 1028, 128)), INVALID),
    (dict(v_strides=(1 << 31, 1024, 128)), INVALID), (dict(k_strides=(-16384, 1024, 128)), INVALID),
    (dict(dtype="f32", k_strides=(16384, 1028, 128)), dck.DCK_OK),
])
def test_descriptors(kw, expect):
    assert dck.dck_validate_paged_desc(_cache(**kw)) == expect


def test_null_descriptor_and_unknown_type():
    assert dck.lib().dck_validate_paged_desc(None) == INVALID
    c = _cache()
    c.desc.dtype = 7
    assert dck.dck_validate_paged_desc(c) == INVALID


def test_page_update_arguments():
    names = ("batch", "page_size", "n_pages", "old_len", "new_len", "seq_len", "block_table", "table_stride", "free_pages",
             "free_in", "free_out", "n_tok", "slots", "positions", "cu_new")
    good = dict(zip(names, (2, 16, 10, A, A, A, A, 4, A, A, A, 5, A, A, A)))

    def call(**kw):
        a = dict(good, **kw)
        return dck.dck_page_update(*[a[n] for n in names], stream=0)
    for kw in (dict(batch=-1), dict(batch=4097), dict(page_size=0), dict(n_pages=0), dict(table_stride=-1),
               dict(table_stride=1 << 31), dict(n_tok=-1), dict(n_tok=1 << 31), dict(old_len=A + 2), dict(slots=A + 4),
               *[{n: None} for n in names if good[n] == A]):
        assert call(**kw) == INVALID, kw
    assert call(page_size=65537) == UNSUPPORTED


def test_rope_arguments():
    names = ("rope", "x", "n_tok", "n_heads", "head_dim", "dtype", "x_token_stride", "x_head_stride", "positions", "out",
             "out_token_stride", "out_head_stride")
    good = dict(zip(names, (dck.Rope(64, 1e4), A, 3, 2, 64, 0, 128, 64, A, 2 * A, 128, 64)))

    def call(**kw):
        a = dict(good, **kw)
        return dck.dck_rope(*[a[n] for n in names], stream=0)
    bad = dck.Rope(64, 1e4)
    bad.table.initialised = 0
    for kw in (dict(n_tok=-1), dict(n_heads=-1), dict(head_dim=62), dict(dtype=3), dict(x=None), dict(out=None),
               dict(positions=None), dict(x=A + 1), dict(positions=A + 2), dict(x_token_stride=-1),
               dict(out_head_stride=32), dict(out_token_stride=10), dict(out=A, out_token_stride=256), dict(rope=bad)):
        assert call(**kw) == INVALID, kw
    assert call(head_dim=65537) == UNSUPPORTED
    assert call(n_tok=0) == call(n_heads=0) == dck.DCK_OK


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=3), dict(rotary_dim=0), dict(theta=0.0), dict(theta=math.inf), dict(theta=math.nan), dict(magnitude=math.nan),
    dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=math.nan), dict(rotary_dim=2, scaling="ntk", factor=2.0),
    dict(scaling="bands", factor=2.0, slow=4.0, fast=4.0, trained_len=10), dict(scaling="bands", factor=2.0, trained_len=0),
    dict(scaling="yarn", factor=2.0, slow=0.0, trained_len=10), dict(scaling="yarn", factor=2.0, theta=1.0, trained_len=10),
    dict(rotary_dim=258),
])
def test_rope_settings_refused(kw):
    a = dict(rotary_dim=64, theta=1e4)
    a.update(kw)
    with pytest.raises(dck.DckError):
        dck.Rope(a.pop("rotary_dim"), a.pop("theta"), **a)


@pytest.mark.parametrize("setting", ROPES + [dict(rotary_dim=256, theta=1e4),
                                             dict(rotary_dim=128, theta=0.01)],
                         ids=lambda s: f"{s.get('scaling', 'none')}{s['rotary_dim']}")
def test_rope_frequencies(setting):
    """turns = w / 2 pi mod 1 as 64-bit fractions: pow, log and the mix round to a double each, so 2^-49 relative."""
    s = dict(setting)
    t = dck.Rope(s.pop("rotary_dim"), s.pop("theta"), **s).table
    s = {k: v for k, v in s.items() if k not in ("layout", "magnitude")}
    w = P.rope_frequencies(setting["rotary_dim"], setting["theta"], **s) / (2 * math.pi)
    got = np.array([t.turns[i] / 2.0 ** 64 for i in range(setting["rotary_dim"] // 2)])
    off = np.abs(got - w % 1.0)
    off = np.minimum(off, 1 - off)
    assert (off <= w * 2.0 ** -49 + 2.0 ** -62).all()
    assert all(t.turns[i] == 0 for i in range(setting["rotary_dim"] // 2, 128))
    assert t.rotary_dim == setting["rotary_dim"] and t.magnitude == np.float32(setting.get("magnitude", 1.0))


def test_append_arguments():
    names = ("cache", "rope", "q", "q_stride", "k", "k_stride", "v", "v_stride", "n_tok", "positions", "slots", "q_out",
             "kcache", "vcache")
    good = dict(zip(names, (_cache(), dck.Rope(128, 1e4), A, 6144, A, 6144, A, 6144, 4, A, A, 2 * A, A, A)))

    def call(**kw):
        a = dict(good, **kw)
        return dck.dck_paged_append(*[a[n] for n in names], stream=0)
    for kw in (dict(n_tok=-1), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None), dict(q_out=None),
               dict(kcache=None), dict(vcache=None), dict(kcache=A + 8), dict(k=A + 1), dict(slots=A + 4),
               dict(k_stride=-1), dict(q_stride=-1), dict(q=2 * A), dict(rope=dck.Rope(256, 1e4)), dict(cache=_cache(page_size=0))):
        assert call(**kw) == INVALID, kw
    assert call(cache=_cache(head_dim=100)) == UNSUPPORTED
    assert call(n_tok=0) == dck.DCK_OK


def test_decode_arguments():
    names = ("cache", "q", "q_stride", "kcache", "vcache", "block_table", "table_stride", "seq_len", "batch", "max_seq_len",
             "scale", "window", "softcap", "out", "lse", "workspace", "ws_bytes")
    good = dict(zip(names, (_cache(), A, 4096, A, A, A, 8, A, 2, 100, 0.1, 0, 0.0, A, None, A, 1 << 40)))

    def call(**kw):
        a = dict(good, **kw)
        return dck.dck_paged_decode_attention(*[a[n] for n in names], stream=0)
    for kw in (dict(batch=-1), dict(batch=4097), dict(max_seq_len=0), dict(window=-1), dict(scale=math.inf),
               dict(scale=math.nan), dict(softcap=-1.0), dict(softcap=math.nan), dict(table_stride=-1), dict(q_stride=-1),
               dict(q=None), dict(kcache=None), dict(vcache=None), dict(block_table=None), dict(seq_len=None),
               dict(out=None), dict(q=A + 1), dict(kcache=A + 8), dict(lse=A + 2), dict(seq_len=A + 1),
               dict(cache=_cache(n_q_heads=31))):
        assert call(**kw) == INVALID, kw
    assert call(cache=_cache(head_dim=12)) == UNSUPPORTED
    assert call(batch=0) == dck.DCK_OK


def test_from_tensors():
    import torch
    both = torch.zeros((5, 2, 16, 8, 128), dtype=torch.bfloat16)
    c = dck.PagedCache.from_tensors(both[:, 0], both[:, 1], 32).desc
    assert (c.n_pages, c.page_size, c.n_kv_heads, c.head_dim, c.n_q_heads) == (5, 16, 8, 128, 32)
    assert (c.k_page_stride, c.k_token_stride, c.k_head_stride) == (2 * 16 * 1024, 1024, 128)
    h = torch.zeros((5, 8, 16, 128)).transpose(1, 2)
    c = dck.PagedCache.from_tensors(h, h, 8).desc
    assert c.dtype == dck.DCK_F32 and (c.v_page_stride, c.v_token_stride, c.v_head_stride) == (16384, 128, 2048)
    for k, v in ((both[:, 0], both[:, 0, :, :, :64]), (both[:, 0].half(), both[:, 1].half()), (both, both),
                 (both[:, 0].transpose(2, 3), both[:, 1].transpose(2, 3))):
        with pytest.raises(ValueError):
            dck.PagedCache.from_tensors(k, v, 32)


def test_page_program_by_hand():
    """The sequential definition on a case written out: page size 4, free list [7, 5, 9]."""
    table = [[1, 2, -1, -1], [3, 4, 6, -1], [-1] * 4]
    # request 0 grows 7 -> 10 (one page), 1 shrinks 12 -> 5 (gives back page 6), 2 starts with 9 (three pages)
    r = P.page_update(4, [7, 12, 0], [10, 5, 9], table, [7, 5, 9, 0, 0], 3, 13)
    assert r["block_table"].tolist() == [[1, 2, 6, -1], [3, 4, 6, -1], [9, 5, 7, -1]]
    assert r["free"].tolist() == [0, 0] and r["seq_len"].tolist() == [10, 5, 9] and r["cu_new"].tolist() == [0, 3, 3, 12]
    assert r["slots"].tolist() == [11, 24, 25, 36, 37, 38, 39, 20, 21, 22, 23, 28, -1]
    assert r["positions"].tolist() == [7, 8, 9] + list(range(9)) + [0]


def test_attention_definition_against_torch():
    import torch
    rng = np.random.default_rng(0)
    kc, vc = rng.standard_normal((2, 6, 4, 2, 16))
    q = rng.standard_normal((2, 4, 16))
    table, lens = np.array([[3, 0, 5], [1, 2, 4]]), [11, 6]
    out, lse, _, _ = P.paged_decode(q, kc, vc, table, lens, 0.25, window=7)
    for b, n in enumerate(lens):
        k, v = (torch.from_numpy(c[table[b]].reshape(12, 2, 16)[max(0, n - 7):n]) for c in (kc, vc))
        k, v = (t.transpose(0, 1).repeat_interleave(2, 0) for t in (k, v))
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[b])[:, None], k, v, scale=0.25)[:, 0]
        assert np.allclose(out[b], want.numpy(), atol=1e-12)
        s = torch.einsum("jd,jtd->jt", torch.from_numpy(q[b]), k) * 0.25
        assert np.allclose(lse[b], torch.logsumexp(s, -1).numpy(), atol=1e-12)
