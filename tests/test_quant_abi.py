"""The 8-bit cache's and the shared attention's entry points refuse what they cannot take, before any CUDA call (fake
aligned addresses, never dereferenced); the definition of 8-bit rows on cases written out."""

import math

import numpy as np
import pytest

from oracle import paged as P
from paper_2607_24331_gb300 import dck

A = 1 << 20  # an aligned address that nothing reads
INVALID, UNSUPPORTED = dck.DCK_ERR_INVALID, dck.DCK_ERR_UNSUPPORTED


def _cache(**kw):
    a = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, dtype="bf16")
    a.update(kw)
    return dck.QuantCache(**a)


@pytest.mark.parametrize("kw,expect", [
    (dict(), dck.DCK_OK), (dict(dtype="f32"), dck.DCK_OK),
    (dict(head_dim=80), dck.DCK_OK), (dict(head_dim=8), INVALID),  # dense heads of 8 bytes: strides off 16
    (dict(head_dim=8, k_strides=(2048, 128, 16), v_strides=(2048, 128, 16)), dck.DCK_OK),
    (dict(n_q_heads=30), INVALID), (dict(n_pages=0), INVALID), (dict(head_dim=100), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(page_size=65537), UNSUPPORTED), (dict(k_strides=(16384, 1032, 128)), INVALID), (dict(v_strides=(16384, 1024, 0)), INVALID),
    (dict(k_scale_strides=(128, 8, 0)), INVALID), (dict(v_scale_strides=(-128, 8, 1)), INVALID),
    (dict(v_scale_strides=(1 << 30, 8, 1)), INVALID), (dict(k_scale_strides=(1, 1, 1)), dck.DCK_OK),
])
def test_descriptors(kw, expect):
    assert dck.dck_validate_quant_desc(_cache(**kw)) == expect


def test_null_descriptor_and_unknown_type():
    assert dck.lib().dck_validate_quant_desc(None) == INVALID
    c = _cache()
    c.desc.cache.dtype = 7
    assert dck.dck_validate_quant_desc(c) == INVALID


def _refusals(f, names, good, invalid, **more):
    def call(**kw):
        a = dict(good, **kw)
        return f(*[a[n] for n in names], stream=0)
    for kw in invalid:
        assert call(**kw) == INVALID, kw
    return call


def test_append_arguments():
    names = ("cache", "rope", "q", "q_stride", "k", "k_stride", "v", "v_stride", "n_tok", "positions", "slots", "q_out",
             "kcache", "k_scale", "vcache", "v_scale")
    good = dict(zip(names, (_cache(), dck.Rope(128, 1e4), A, 6144, A, 6144, A, 6144, 4, A, A, 2 * A, A, A, A, A)))
    call = _refusals(dck.dck_quant_append, names, good, [
        dict(n_tok=-1), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None), dict(q_out=None), dict(kcache=None),
        dict(vcache=None), dict(k_scale=None), dict(v_scale=None), dict(k_scale=A + 2), dict(v_scale=A + 1), dict(kcache=A + 8),
        dict(k=A + 1), dict(slots=A + 4), dict(k_stride=-1), dict(q_stride=-1), dict(q=2 * A), dict(rope=dck.Rope(256, 1e4)),
        dict(cache=_cache(page_size=0))])
    assert call(cache=_cache(head_dim=100)) == UNSUPPORTED
    assert call(n_tok=0) == dck.DCK_OK


def test_read_arguments():
    names = ("cache", "n_tok", "slots", "kcache", "k_scale", "vcache", "v_scale", "k", "k_stride", "v", "v_stride")
    good = dict(zip(names, (_cache(), 3, A, A, A, A, A, A, 1024, A, 1024)))
    call = _refusals(dck.dck_quant_read, names, good, [
        dict(n_tok=-1), *[{n: None} for n in names if good[n] == A and n != "cache"], dict(slots=A + 4), dict(kcache=A + 8),
        dict(k_scale=A + 2), dict(k=A + 1), dict(k_stride=1023), dict(v_stride=-1), dict(v_stride=1 << 31),
        dict(cache=_cache(n_pages=0))])
    assert call(n_tok=0) == dck.DCK_OK
    assert call(cache=_cache(page_size=1 << 17)) == UNSUPPORTED


ATTEND = ("table", "table_stride", "seq_len", "batch", "max_seq_len")
BAD = [dict(batch=-1), dict(batch=4097), dict(max_seq_len=0), dict(window=-1), dict(scale=math.inf), dict(scale=math.nan),
       dict(softcap=-1.0), dict(softcap=math.nan), dict(table_stride=-1), dict(q_stride=-1), dict(q=None), dict(kcache=None),
       dict(vcache=None), dict(table=None), dict(seq_len=None), dict(out=None), dict(q=A + 1), dict(kcache=A + 8),
       dict(lse=A + 2), dict(seq_len=A + 1)]
SCALES = [dict(k_scale=None), dict(v_scale=None), dict(k_scale=A + 2)]
GROUPS = [dict(max_own=0), dict(n_groups=-1), dict(n_groups=0), dict(n_groups=3), dict(group_start=None), dict(shared_len=None),
          dict(group_start=A + 2), dict(shared_len=A + 1)]


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_attention_arguments(quant, shared):
    caches = ("kcache", "k_scale", "vcache", "v_scale") if quant else ("kcache", "vcache")
    names = ("cache", "q", "q_stride", *caches, *ATTEND, *(("max_own", "n_groups", "group_start", "shared_len") if shared else ()),
             "scale", "window", "softcap", "out", "lse", "workspace", "ws_bytes")
    good = dict(q_stride=4096, table_stride=8, batch=2, max_seq_len=100, max_own=50, n_groups=2, scale=0.1, window=0,
                softcap=0.0, lse=None, ws_bytes=1 << 40,
                cache=_cache() if quant else dck.PagedCache(32, 8, 128, 16, 100, "bf16"))
    good = {n: good.get(n, A) for n in names} | dict(lse=None)
    f = {(False, True): dck.dck_paged_shared_attention, (True, True): dck.dck_quant_shared_attention,
         (True, False): dck.dck_quant_decode_attention, (False, False): dck.dck_paged_decode_attention}[quant, shared]
    call = _refusals(f, names, good, BAD + (SCALES if quant else []) + (GROUPS if shared else []))
    assert call(batch=0, **(dict(n_groups=0) if shared else {})) == dck.DCK_OK


def test_workspace_sizes_of_bad_arguments_are_zero():
    c = dck.PagedCache(32, 8, 128, 16, 100, "bf16")
    for args in ((-1, 100, 10), (4097, 100, 10), (4, 0, 10), (4, 100, 0)):
        assert dck.dck_paged_shared_workspace_size(c, *args) == dck.dck_quant_shared_workspace_size(_cache(), *args) == 0
    assert dck.dck_quant_decode_workspace_size(_cache(n_pages=0), 4, 100) == 0


def test_way_of_shared_calls():
    assert dck.dck_set_shared_way(2) == 0 and dck.dck_set_shared_way(7) == 2 and dck.dck_set_shared_way(-1) == 2
    assert dck.dck_set_shared_way(0) == 2


def test_from_tensors():
    import torch
    both, scales = torch.zeros((5, 2, 16, 8, 128), dtype=torch.uint8), torch.zeros((5, 16, 2, 8))
    c = dck.QuantCache.from_tensors(both[:, 0], scales[:, :, 0], both[:, 1], scales[:, :, 1], 32, "f32").desc
    assert (c.cache.n_pages, c.cache.page_size, c.cache.n_kv_heads, c.cache.head_dim, c.cache.dtype) == (5, 16, 8, 128, dck.DCK_F32)
    assert (c.cache.k_page_stride, c.cache.k_token_stride, c.cache.k_head_stride) == (2 * 16 * 1024, 1024, 128)
    assert (c.k_scale_page_stride, c.v_scale_token_stride, c.v_scale_head_stride) == (256, 16, 1)
    f8 = both.view(torch.float8_e4m3fn)
    assert dck.QuantCache.from_tensors(f8[:, 0], scales[:, :, 0], f8[:, 1], scales[:, :, 1], 8, "bf16").desc.cache.dtype == dck.DCK_BF16
    s = scales[:, :, 0]
    for args in ((both[:, 0].short(), s, both[:, 1], s, 32, "bf16"), (both[:, 0], s[:, :, :7], both[:, 1], s, 32, "bf16"),
                 (both[:, 0], s.double(), both[:, 1], s, 32, "bf16"), (both[:, 0], s, both[:, 1], s, 32, "fp16"),
                 (both[:, 0].transpose(2, 3), s, both[:, 1].transpose(2, 3), s, 32, "bf16")):
        with pytest.raises(ValueError):
            dck.QuantCache.from_tensors(*args)


def test_eight_bit_rows_by_hand():
    v = P.code_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1 and v[0x7e] == 448 and v[0xfe] == -448
    assert math.isnan(v[0x7f]) and math.isnan(v[0xff])
    codes, scales = P.quantise([[448.0, -1.0, 17.0, 19.0], [449.0, 0.0, -0.0, 2.0 ** -10], [0.0, 0.0, 0.0, 0.0],
                                [math.inf, math.nan, 0.25, -0.4375]])
    # 17 and 19 lie half way between 16, 18 and 20
    assert scales.tolist() == [1.0, 2.0, 2.0 ** -126, 2.0 ** -10]
    assert P.stand_for(codes, scales)[0].tolist() == [448.0, -1.0, 16.0, 20.0]
    assert P.stand_for(codes, scales)[1].tolist() == [448.0, 0.0, -0.0, 0.0]  # 224.5 to 224; 2^-11 to 0, even
    assert np.isnan(P.stand_for(codes, scales)[3][:2]).all() and P.stand_for(codes, scales)[3][2:].tolist() == [0.25, -0.4375]


def test_eight_bit_rows_against_torch():
    import torch
    x = np.random.default_rng(1).standard_normal((20, 3, 64)) * 10.0 ** np.arange(-10, 10)[:, None, None]
    codes, scales = P.quantise(x)
    assert ((np.abs(x).max(-1) <= 448 * scales) & (np.abs(x).max(-1) > 224 * scales)).all()
    want = torch.from_numpy(x / scales[..., None]).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    near = np.abs(x / scales[..., None] - P.code_values()[codes])
    assert (near <= np.maximum(np.abs(x / scales[..., None]) * 2.0 ** -4, 2.0 ** -10)).all()
    assert (codes == want).mean() > 0.9999  # (the quotients are rounded to 32 bits for torch)
