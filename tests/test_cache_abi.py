"""What the cache's and attention's entry points refuse, before any launch (no GPU: the pointers are never followed)."""
import ctypes

import pytest

import paper_2501_16385_amd as fbq
from paper_2501_16385_amd.cache import _CAttentionCall, _CCache, _CCacheDesc

OK, ODD2, ODD8 = 0x10000, 0x10002, 0x10008


def desc(**over):
    d = dict(layers=2, pages=8, page_size=16, kv_heads=2, head_dim=64, type=0)
    d.update(over)
    return _CCacheDesc(*[d[n] for n, _ in _CCacheDesc._fields_])


def cache(d=None, **over):
    c = dict(rows=4, max_pages=6, pool=OK, table=OK, lengths=OK, refs=OK)
    c.update(over)
    return _CCache(d or desc(), *[c[n] for n, _ in _CCache._fields_[1:]])


def call(c=None, **over):
    a = dict(layer=0, heads=4, T=4, max_q=1, q_start=None, q=OK, q_stride=256, out=OK, out_stride=256, lse=None, shared=None, n_shared=0, scale=1.0)
    a.update(over)
    return _CAttentionCall(c or cache(), *[a[n] for n, _ in _CAttentionCall._fields_[1:]])


BAD_DESCS = [(dict(layers=0), 2), (dict(pages=0), 2), (dict(pages=(1 << 22) + 1), 2), (dict(kv_heads=0), 2), (dict(head_dim=8), 2), (dict(head_dim=264), 2), (dict(head_dim=68), 2),
             (dict(page_size=8), 3), (dict(page_size=48), 3), (dict(page_size=512), 3), (dict(type=2), 3), (dict(type=-1), 3)]
BAD_CACHES = [(dict(rows=0), 2), (dict(rows=65537), 2), (dict(max_pages=0), 2), (dict(max_pages=(1 << 20) + 1), 3), (dict(rows=65536, max_pages=1 << 20), 3),
              (dict(pool=None), 1), (dict(table=None), 1), (dict(lengths=None), 1), (dict(pool=ODD8), 4), (dict(table=ODD2), 4), (dict(lengths=ODD2), 4)]


def every_entry(lib, c):
    """(entry point, status) of each for the cache c, everything else in order."""
    r = ctypes.byref(c)
    return {"reserve": lib.fbq_cache_reserve(r, OK, OK, None, None), "append": lib.fbq_cache_append(r, 0, 4, None, OK, OK, 128, OK, 128, None),
            "free": lib.fbq_cache_free(r, 1, OK, None), "fork": lib.fbq_cache_fork(r, 1, OK, OK, None, OK, 1 << 20, None),
            "copy": lib.fbq_cache_copy(r, 1, OK, OK, None), "compact": lib.fbq_cache_compact(r, OK, OK, None, OK, 1 << 30, None),
            "attention": lib.fbq_attention(ctypes.byref(call(c)), OK, 1 << 40, None)}


@pytest.mark.parametrize("over,code", BAD_DESCS)
def test_descriptors(over, code):
    lib = fbq.load()
    d = desc(**over)
    assert lib.fbq_check_cache(ctypes.byref(d)) == code
    assert lib.fbq_cache_bytes(ctypes.byref(d)) == 0 and lib.fbq_cache_workspace_bytes(ctypes.byref(d), 1) == 0
    assert lib.fbq_attention_workspace_bytes(ctypes.byref(call(cache(d)))) == 0
    assert set(every_entry(lib, cache(d)).values()) == {code}


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_caches(over, code):
    assert set(every_entry(fbq.load(), cache(**over)).values()) == {code}


def test_sizes():
    lib = fbq.load()
    d = desc()
    assert lib.fbq_check_cache(ctypes.byref(d)) == 0 and lib.fbq_check_cache(None) == 1
    assert lib.fbq_cache_bytes(ctypes.byref(d)) == 2 * 8 * 2 * 2 * 16 * 64 * 2
    assert lib.fbq_cache_workspace_bytes(ctypes.byref(d), 5) >= 5 * 8 and lib.fbq_cache_workspace_bytes(ctypes.byref(d), 0) >= 3 * 8 * 4
    assert lib.fbq_cache_workspace_bytes(ctypes.byref(d), -1) == 0
    assert lib.fbq_attention_workspace_bytes(ctypes.byref(call())) == 0          # rows of at most 96 tokens: nothing to join
    wide = call(cache(max_pages=64))
    assert lib.fbq_attention_workspace_bytes(ctypes.byref(wide)) > 0 and lib.fbq_attention_workspace_bytes(None) == 0
    bare = call(cache(max_pages=64, pool=None, table=None, lengths=None, refs=None), q=None, out=None)
    assert lib.fbq_attention_workspace_bytes(ctypes.byref(bare)) == lib.fbq_attention_workspace_bytes(ctypes.byref(wide))     # pointers are not looked at


def test_page_operations():
    lib = fbq.load()
    r, no_refs = ctypes.byref(cache()), ctypes.byref(cache(refs=None))
    for f in (lib.fbq_cache_reserve, ):
        assert f(None, OK, OK, None, None) == 1 and f(r, None, OK, None, None) == 1 and f(r, OK, None, None, None) == 1 and f(no_refs, OK, OK, None, None) == 1
        assert f(r, ODD2, OK, None, None) == 4 and f(r, OK, ODD2, None, None) == 4 and f(r, OK, OK, ODD2, None) == 4
    append = lambda layer=0, T=4, qs=None, start=OK, k=OK, ks=128, v=OK, vs=128: lib.fbq_cache_append(r, layer, T, qs, start, k, ks, v, vs, None)
    assert append(layer=2) == append(layer=-1) == append(T=0) == append(T=3) == append(T=(1 << 24) + 1, qs=OK) == 2
    assert append(ks=120) == append(vs=127) == append(ks=132) == append(vs=1 << 33) == 2
    assert append(start=None) == append(k=None) == append(v=None) == 1
    assert append(k=ODD8) == append(v=ODD8) == append(start=ODD2) == append(qs=ODD2) == 4
    free = lambda n, rows: lib.fbq_cache_free(r, n, rows, None)
    assert free(0, OK) == free(65537, OK) == 2 and free(1, None) == 1 and free(1, ODD2) == 4
    fork = lambda n=2, a=OK, b=OK, info=None, ws=OK, size=16: lib.fbq_cache_fork(r, n, a, b, info, ws, size, None)
    assert fork(n=0) == fork(n=65537) == 2 and fork(a=None) == fork(b=None) == fork(ws=None) == 1
    assert fork(a=ODD2) == fork(b=ODD2) == fork(info=ODD2) == fork(ws=ODD8) == 4 and fork(size=15) == 5
    copy = lambda n=1, a=OK, b=OK: lib.fbq_cache_copy(r, n, a, b, None)
    assert copy(n=0) == 2 and copy(a=None) == copy(b=None) == 1 and copy(a=ODD2) == copy(b=ODD2) == 4
    compact = lambda t=OK, f=OK, info=None, ws=OK, size=1 << 20: lib.fbq_cache_compact(r, t, f, info, ws, size, None)
    assert compact(t=None) == compact(f=None) == compact(ws=None) == 1 and compact(t=ODD2) == compact(f=ODD2) == compact(info=ODD2) == compact(ws=ODD8) == 4
    assert compact(size=fbq.load().fbq_cache_workspace_bytes(ctypes.byref(desc()), 0) - 1) == 5


def test_attention():
    lib = fbq.load()
    go = lambda ws=OK, size=1 << 40, **over: lib.fbq_attention(ctypes.byref(call(cache(max_pages=64), **over)), ws, size, None)
    assert lib.fbq_attention(None, OK, 1 << 40, None) == 1
    for bad in (dict(layer=2), dict(layer=-1), dict(heads=0), dict(heads=3), dict(T=0), dict(T=3), dict(max_q=2), dict(max_q=0), dict(q_start=OK, T=9, max_q=10), dict(n_shared=-1),
                dict(n_shared=65, shared=OK), dict(q_stride=248), dict(out_stride=255), dict(q_stride=260)):
        assert go(**bad) == 2, bad
        assert lib.fbq_attention_workspace_bytes(ctypes.byref(call(cache(max_pages=64), **bad))) == 0, bad
    assert go(heads=16384, q_stride=1 << 20, out_stride=1 << 20) == go(q_start=OK, T=(1 << 20) + 1, max_q=5) == go(q_stride=1 << 33) == 3
    assert go(q=None) == go(out=None) == go(n_shared=2) == go(ws=None) == 1
    assert go(q=ODD8) == go(out=ODD8) == go(lse=ODD2) == go(q_start=ODD2, T=8, max_q=3) == go(shared=ODD2, n_shared=1) == go(ws=ODD8) == 4
    assert go(size=lib.fbq_attention_workspace_bytes(ctypes.byref(call(cache(max_pages=64)))) - 1) == 5


def test_the_binding_refuses_tensors_that_are_not_as_they_should_be():
    import torch
    pool, table, ints = torch.zeros(1, 4, 2, 2, 16, 64, dtype=torch.float16), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        fbq.Cache(pool, table, ints, ints)                      # host tensors
    with pytest.raises(ValueError):
        fbq.Cache(pool.float(), table, ints, ints)
    with pytest.raises(ValueError):
        fbq.Cache(pool[0], table, ints, ints)
    with pytest.raises(ValueError):
        fbq.Cache(pool, table[0], ints, ints)
