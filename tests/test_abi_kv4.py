"""Refusals of the 4-bit cache's entry points, before any HIP call (no GPU)."""
import ctypes

import pytest
import torch

import paper_2609_32420_amd as P
from paper_2609_32420_amd import build as B

PTR = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10002)


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(P.LIB_PATH):
        B.build()
    return P.lib()


def _cache(pages=0x100000, n=4, heads=2, d=128, block=64):
    return P.Kv4(pages, n, heads, d, block)


def _rows(data=0x200000, st=256, sh=128):
    return P.Rows(data, st, sh)


BAD_CACHES = [(dict(pages=0), -1), (dict(n=0), -2), (dict(heads=0), -2), (dict(d=96), -3), (dict(block=32), -3),
              (dict(n=1 << 25, block=64), -2), (dict(heads=65536), -3), (dict(pages=0x100008), -4)]


def test_page_bytes(L):
    assert L.carnator_kv4_page_bytes(1, 64, 64) == 64 * 64 * 17 // 16
    assert L.carnator_kv4_page_bytes(12, 128, 128) == 12 * 17408
    for bad in ((0, 64, 64), (1, 96, 64), (1, 64, 32), (65536, 64, 64)):
        assert L.carnator_kv4_page_bytes(*bad) == 0


def _plan(L, kv=PTR, new=PTR, batch=2, table=PTR, width=3, free=PTR, n_free=4, block=64, q=PTR,
          out=ctypes.c_void_p(0x30000), slots=PTR, pos=None, n=5, counts=PTR):
    return L.carnator_page_plan(kv, new, batch, table, width, free, n_free, block, q, out, slots, pos, n, counts, None)


@pytest.mark.parametrize("change,code", [
    (dict(kv=None), -1), (dict(new=None), -1), (dict(table=None), -1), (dict(free=None), -1), (dict(q=None), -1),
    (dict(out=None), -1), (dict(slots=None), -1), (dict(counts=None), -1), (dict(batch=0), -2), (dict(width=0), -2),
    (dict(n_free=-1), -2), (dict(n=-1), -2), (dict(out=PTR), -2), (dict(width=(1 << 24) + 1), -2),
    (dict(block=96), -3), (dict(batch=16385), -3), (dict(slots=ODD), -4), (dict(pos=ODD), -4), (dict(table=ODD), -4)])
def test_plan_rejects(L, change, code):
    assert _plan(L, **change) == code and L.carnator_last_error()


def _store(L, cache=None, k=None, v=None, n=3, slots=PTR):
    c = _cache() if cache is None else cache
    k, v = _rows() if k is None else k, _rows() if v is None else v
    return L.carnator_kv4_store(ctypes.byref(c), ctypes.byref(k), ctypes.byref(v), n, slots, None)


def test_store_rejects(L):
    for change, code in BAD_CACHES:
        assert _store(L, cache=_cache(**change)) == code
    for bad, code in ((_rows(data=0), -1), (_rows(data=0x200008), -4), (_rows(st=260), -4), (_rows(sh=4), -4),
                      (_rows(st=-256), -2), (_rows(sh=-128), -2)):
        assert _store(L, k=bad) == code and _store(L, v=bad) == code
    assert _store(L, n=-1) == -2 and _store(L, slots=None) == -1 and _store(L, slots=ODD) == -4
    assert L.carnator_kv4_store(None, ctypes.byref(_rows()), ctypes.byref(_rows()), 3, PTR, None) == -1
    # nothing to store: nothing is looked at
    assert _store(L, k=_rows(data=0), v=_rows(data=0), n=0, slots=None) == 0


def _load(L, cache=None, table=PTR, batch=2, width=3, kv=PTR, n=100, ko=0x40000, ks=(25600, 12800, 128), vo=0x50000,
          vs=(25600, 12800, 128)):
    c = _cache() if cache is None else cache
    return L.carnator_kv4_load(ctypes.byref(c), table, batch, width, kv, n, ko, *ks, vo, *vs, None)


def test_load_rejects(L):
    for change, code in BAD_CACHES:
        assert _load(L, cache=_cache(**change)) == code
    for change, code in ((dict(table=None), -1), (dict(kv=None), -1), (dict(ko=None), -1), (dict(vo=None), -1),
                         (dict(batch=0), -2), (dict(width=0), -2), (dict(n=-1), -2), (dict(width=(1 << 24) + 1), -2),
                         (dict(ks=(25600, 12800, 64)), -2), (dict(vs=(-8, 12800, 128)), -2),
                         (dict(ks=(25600, 12800, 132)), -4), (dict(ko=0x40008), -4), (dict(vo=0x50008), -4),
                         (dict(table=ODD), -4), (dict(kv=ODD), -4)):
        assert _load(L, **change) == code, change
    assert _load(L, n=0, ko=None, vo=None) == 0


def _attn(L, q=None, rows=6, heads=4, cache=None, table=PTR, batch=2, width=3, start=PTR, kv=PTR, most=3, scale=0.0,
          out=0x60000, ost=512, osh=128, lse=None, ws=0x70000, size=1 << 30):
    c, q = _cache() if cache is None else cache, _rows(st=512) if q is None else q
    return L.carnator_kv4_attn(ctypes.byref(q), rows, heads, ctypes.byref(c), table, batch, width, start, kv, most, 1,
                               scale, out, ost, osh, lse, ws, size, None)


def test_attention_rejects(L):
    for change, code in BAD_CACHES:
        assert _attn(L, cache=_cache(**change)) == code
    for change, code in ((dict(q=_rows(data=0)), -1), (dict(table=None), -1), (dict(start=None), -1), (dict(kv=None), -1),
                         (dict(out=None), -1), (dict(heads=3), -2), (dict(heads=0), -2), (dict(rows=-1), -2),
                         (dict(batch=0), -2), (dict(width=0), -2), (dict(most=0), -2), (dict(scale=float("nan")), -2),
                         (dict(scale=float("inf")), -2), (dict(ost=64), -2), (dict(osh=64), -2),
                         (dict(width=(1 << 24) + 1), -2), (dict(rows=1 << 30), -2), (dict(q=_rows(st=4)), -4),
                         (dict(q=_rows(data=0x200008)), -4), (dict(out=0x60008), -4), (dict(ost=516), -4),
                         (dict(lse=ODD), -4), (dict(table=ODD), -4), (dict(start=ODD), -4)):
        assert _attn(L, **change) == code, change
    # more workgroups than a launch holds
    assert _attn(L, batch=1 << 25) == -3
    assert _attn(L, rows=0, q=_rows(data=0), out=None) == 0


def test_attention_workspace(L):
    size = lambda c, *a: L.carnator_kv4_attn_workspace_size(ctypes.byref(c), *a)  # noqa: E731
    assert size(_cache(d=96), 4, 6, 2, 3, 3) == 0 and size(_cache(), 3, 6, 2, 3, 3) == 0
    assert size(_cache(), 4, 0, 2, 3, 3) == 0
    # a long cache and few rows: parts of the key axis are joined through it
    need = size(_cache(n=100), 4, 2, 2, 2000, 1)
    if need:
        assert _attn(L, cache=_cache(n=100), rows=2, width=2000, most=1, size=need - 1) == -5
        assert _attn(L, cache=_cache(n=100), rows=2, width=2000, most=1, ws=None) == -5
        assert _attn(L, cache=_cache(n=100), rows=2, width=2000, most=1, ws=0x70010) == -4


def test_binding_rejects():
    cpu = torch.zeros(2, 2, 64 * 128 * 17 // 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        P.kv4_store(cpu, torch.zeros(1, 2, 128), torch.zeros(1, 2, 128), torch.zeros(1, dtype=torch.int32), 64)
    with pytest.raises(ValueError):
        P.kv4_load(cpu, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 64)
    with pytest.raises(ValueError):
        P.page_plan(torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                    torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 64, 1)
    for bad in ((1, 2, 96, 64), (1, 2, 64, 32), (1, 0, 64, 64)):
        with pytest.raises(ValueError):
            P.kv4_pool(*bad, device="cpu")
