"""Host-side checks of the entry points that run a quantized block (rows to 8 bits, integer projection, paged
cache, attention over it): refusals before any device work, and the workspace size."""
import ctypes

import pytest
import torch

from paper_2609_34866_amd import jab

FAKE = 0x10000      # aligned, never dereferenced


def _prob(**kw):
    base = dict(batch=1, seq_len=8, d_model=64, n_heads=4, n_kv_heads=2, head_dim=64, group_size=32,
                dtype=jab.BF16, scheme=jab.ASYM, rope_theta=0.0)
    base.update(kw)
    return jab.Problem(*[base[k] for k, _ in jab.Problem._fields_])


def _cache(**kw):
    base = dict(bits=8, page_size=64, n_pages=4, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, k_zero=FAKE, v_zero=FAKE)
    base.update(kw)
    return jab._CacheStruct(*[base[k] for k, _ in jab._CacheStruct._fields_])


def _rows(**kw):
    base = dict(n_seq=2, max_pages=2, max_new=4, pages=FAKE, past=FAKE, start=FAKE)
    base.update(kw)
    return jab._CacheRowsStruct(*[base[k] for k, _ in jab._CacheRowsStruct._fields_])


def _calls(p, c, r, y=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    L = jab.lib()
    a = (None if p is None else ctypes.byref(p), None if c is None else ctypes.byref(c),
         None if r is None else ctypes.byref(r))
    return {"write": lambda: L.jab_cache_write(*a, y, None), "read": lambda: L.jab_cache_read(*a, out, out, None),
            "attn": lambda: L.jab_attn_cache(*a, y, out, ws, ws_bytes, None)}


@pytest.mark.parametrize("op", ["write", "read", "attn"])
@pytest.mark.parametrize("c,r,status", [
    (dict(bits=3), {}, jab.JAB_E_INVALID),
    (dict(page_size=16), {}, jab.JAB_E_INVALID),
    (dict(page_size=96), {}, jab.JAB_E_INVALID),
    (dict(page_size=512), {}, jab.JAB_E_INVALID),
    (dict(n_pages=0), {}, jab.JAB_E_INVALID),
    (dict(k=None), {}, jab.JAB_E_INVALID),
    (dict(v=FAKE + 8), {}, jab.JAB_E_INVALID),
    (dict(k_scale=FAKE + 4), {}, jab.JAB_E_INVALID),
    (dict(v_scale=None), {}, jab.JAB_E_INVALID),
    (dict(v_zero=None), {}, jab.JAB_E_INVALID),            # asymmetric: both zero-points
    (dict(k_zero=FAKE + 2), {}, jab.JAB_E_INVALID),
    ({}, dict(n_seq=0), jab.JAB_E_INVALID),
    ({}, dict(max_pages=-1), jab.JAB_E_INVALID),
    ({}, dict(max_new=0), jab.JAB_E_INVALID),
    ({}, dict(pages=None), jab.JAB_E_INVALID),
    ({}, dict(past=FAKE + 2), jab.JAB_E_INVALID),
    ({}, dict(start=None), jab.JAB_E_INVALID),
    (dict(page_size=256), dict(max_pages=1 << 23), jab.JAB_E_UNSUPPORTED),
    ({}, dict(n_seq=(1 << 22) + 1), jab.JAB_E_UNSUPPORTED),
])
def test_cache_refusals(op, c, r, status):
    assert _calls(_prob(), _cache(**c), _rows(**r))[op]() == status
    assert jab.lib().jab_last_error()


@pytest.mark.parametrize("op", ["write", "read", "attn"])
def test_cache_refusals_of_pointers_and_problems(op):
    def status(p=_prob(), c=_cache(), r=_rows(), **kw):
        return _calls(p, c, r, **kw)[op]()

    assert status(p=None) == status(c=None) == status(r=None) == jab.JAB_E_INVALID
    assert status(p=_prob(head_dim=32)) == jab.JAB_E_UNSUPPORTED
    assert status(p=_prob(n_heads=6)) == jab.JAB_E_UNSUPPORTED                # ratio 3
    assert status(p=_prob(scheme=jab.SYM)) == jab.JAB_E_INVALID               # zero-points given
    if op != "read":
        assert status(y=None) == status(y=FAKE + 8) == jab.JAB_E_INVALID
    if op != "write":
        assert status(out=None) == status(out=FAKE + 4) == jab.JAB_E_INVALID


def test_attention_workspace():
    L = jab.lib()

    def size(p, c, r):
        return L.jab_attn_cache_workspace(ctypes.byref(p), ctypes.byref(c), ctypes.byref(r))

    # a short cache is not split and needs none; buffers need not exist yet
    none = dict(k=None, v=None, k_scale=None, v_scale=None, k_zero=None, v_zero=None)
    assert size(_prob(), _cache(**none), _rows(pages=None, past=None, start=None)) == 0
    p, r = _prob(seq_len=1), _rows(n_seq=1, max_pages=512, max_new=1)
    n = size(p, _cache(page_size=256), r)
    assert n >= 2 * 2 * 16 * (64 + 4) * 4                  # two pieces of 16 rows for each share: O, m, l
    # it does not grow with the batch's rows
    assert size(_prob(seq_len=1 << 20), _cache(page_size=256), r) == n
    assert size(_prob(head_dim=32), _cache(), r) == size(p, _cache(bits=5), r) == ctypes.c_size_t(-1).value
    attn = _calls(p, _cache(page_size=256), r, ws_bytes=n - 1)["attn"]
    assert attn() == jab.JAB_E_WORKSPACE
    for ws in (None, FAKE + 128):
        assert _calls(p, _cache(page_size=256), r, ws=ws)["attn"]() == jab.JAB_E_INVALID


def test_rows_and_projection_refusals():
    L, p = jab.lib(), _prob()

    def rows(p=p, n=4, src=FAKE, codes=FAKE, scale=FAKE):
        return L.jab_quant_rows(None if p is None else ctypes.byref(p), n, src, codes, scale, None)

    assert rows(p=None) == rows(n=0) == rows(n=-3) == rows(src=None) == rows(src=FAKE + 8) == jab.JAB_E_INVALID
    assert rows(codes=None) == rows(codes=FAKE + 8) == rows(scale=None) == rows(scale=FAKE + 2) == jab.JAB_E_INVALID
    assert rows(p=_prob(dtype=7)) == jab.JAB_E_UNSUPPORTED

    def project(p=p, xq=FAKE, sx=FAKE, wq=FAKE, sw=FAKE, y=FAKE):
        return L.jab_project_int(ctypes.byref(p), xq, sx, wq, sw, y, None)

    for name in ("xq", "sx", "wq", "sw", "y"):
        assert project(**{name: None}) == jab.JAB_E_INVALID, name
        assert project(**{name: FAKE + 2}) == jab.JAB_E_INVALID, name
    assert project(p=_prob(d_model=131072)) == jab.JAB_E_UNSUPPORTED


def test_binding_refuses_what_the_library_cannot_see():
    p = _prob()
    with pytest.raises(jab.JabError):                      # a CPU tensor
        jab.quant_rows(p, torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(jab.JabError):                      # rows of another length
        jab.quant_rows(p, torch.zeros(4, 32, dtype=torch.bfloat16))
    with pytest.raises(jab.JabError):
        jab.Cache.empty(p, 3, 64, 2, device="cpu")
    with pytest.raises(jab.JabError):
        jab.Cache.empty(p, 8, 48, 2, device="cpu")
    with pytest.raises(jab.JabError):
        jab.CacheRows(torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
                      torch.zeros(5, dtype=torch.int32), 1)
