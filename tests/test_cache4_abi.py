"""What the entry points for a cache in 4 bits, the attention weights and the eviction refuse, before any launch (no GPU: the pointers are never followed), and their kernels' resources."""
import ctypes
import re
from types import SimpleNamespace

import pytest
import torch

import paper_2501_16385_amd as fbq
from paper_2501_16385_amd import cache as kv
from test_cache_abi import BAD_CACHES, BAD_DESCS, ODD2, ODD8, OK, cache, call, desc, every_entry
from test_kernel_resources import code_objects, kernels  # noqa: F401

FOUR = dict(type=4)


def entries(lib, c, rows=4):
    """(entry point, status) of those that came with the cache in 4 bits, everything else in order."""
    r = ctypes.byref(c)
    a = call(c, lse=OK, out=None)
    return {"read": lib.fbq_cache_read(r, 0, rows, None, OK, OK, OK, None), "weights": lib.fbq_attention_weights(ctypes.byref(a), OK, OK, 64, 1.0, None),
            "evict": lib.fbq_cache_evict(r, OK, OK, 1 << 24, 64, OK, 0, 0, None, OK, 1 << 40, None)}


@pytest.mark.parametrize("over,code", BAD_DESCS)
def test_descriptors(over, code):
    lib = fbq.load()
    assert set(entries(lib, cache(desc(**over))).values()) == {code}
    if "type" not in over:
        d = desc(**over, **FOUR)
        assert lib.fbq_check_cache(ctypes.byref(d)) == code and lib.fbq_cache_bytes(ctypes.byref(d)) == 0
        assert set({**every_entry(lib, cache(d)), **entries(lib, cache(d))}.values()) == {code}


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_caches(over, code):
    for d in (desc(), desc(**FOUR)):
        assert set(entries(fbq.load(), cache(d, **over)).values()) == {code}
    assert set(every_entry(fbq.load(), cache(desc(**FOUR), **over)).values()) == {code}


@pytest.mark.parametrize("type_", [2, 3, 6, 7, 8, 12, -4])
def test_types_that_there_are_none_of(type_):
    assert fbq.load().fbq_check_cache(ctypes.byref(desc(type=type_))) == 3


@pytest.mark.parametrize("D,bytes_", [(16, 36), (64, 36), (72, 56), (96, 56), (104, 72), (128, 72), (136, 108), (192, 108), (200, 144), (256, 144)])
def test_bytes(D, bytes_):
    lib = fbq.load()
    assert fbq.token_bytes(D) == bytes_
    for t in (4, 5):
        d = desc(head_dim=D, type=t)
        assert lib.fbq_check_cache(ctypes.byref(d)) == 0 and lib.fbq_cache_bytes(ctypes.byref(d)) == 2 * 8 * 2 * 2 * 16 * bytes_
    c = call(cache(desc(head_dim=D, type=4), max_pages=256), q_stride=4 * D, out_stride=4 * D)
    assert lib.fbq_attention_workspace_bytes(ctypes.byref(c)) > 0


def test_read():
    lib = fbq.load()
    go = lambda layer=0, T=4, qs=None, start=OK, k=OK, v=OK: lib.fbq_cache_read(ctypes.byref(cache(refs=None)), layer, T, qs, start, k, v, None)
    assert go(layer=2) == go(layer=-1) == go(T=0) == go(T=3) == go(T=(1 << 23) + 1, qs=OK) == 2
    assert go(start=None) == go(k=None, v=None) == 1
    assert go(start=ODD2) == go(qs=ODD2) == go(k=ODD8) == go(v=ODD8) == 4


def test_weights():
    lib = fbq.load()
    go = lambda w=OK, out=OK, width=64, decay=1.0, c=None, **over: lib.fbq_attention_weights(ctypes.byref(call(c or cache(refs=None), **{**dict(lse=OK, out=None), **over})), w, out, width, decay, None)
    assert lib.fbq_attention_weights(None, OK, OK, 64, 1.0, None) == 1
    for bad in (dict(layer=2), dict(layer=-1), dict(heads=0), dict(heads=3), dict(T=0), dict(T=3), dict(max_q=2), dict(max_q=0), dict(q_start=OK, T=9, max_q=10), dict(q_stride=248),
                dict(q_stride=260), dict(width=0), dict(width=(1 << 24) + 1), dict(decay=-0.1), dict(decay=1.1), dict(decay=float("nan"))):
        assert go(**bad) == 2, bad
    assert go(heads=16384, q_stride=1 << 20) == go(q_start=OK, T=(1 << 20) + 1, max_q=5) == go(q_stride=1 << 33) == 3
    many = cache(desc(kv_heads=1024, head_dim=16), rows=65536, max_pages=1)
    assert go(c=many, heads=1024, T=65536, q_stride=1024 * 16) == 3
    assert go(out=OK + 64) == go(out=OK - 64) == 3               # one over a part of the other
    assert go(q=None) == go(lse=None) == go(out=None) == 1
    assert go(q=ODD8) == go(lse=ODD2) == go(out=ODD2) == go(w=ODD2) == go(q_start=ODD2, T=8, max_q=3) == 4


def test_evict():
    lib = fbq.load()
    c = cache()
    need = lib.fbq_cache_evict_workspace_bytes(ctypes.byref(c), 64)
    assert need >= 4 * 4 + 2 * 4 * 2 * 64 * 4
    bare = cache(pool=None, table=None, lengths=None, refs=None)
    assert lib.fbq_cache_evict_workspace_bytes(ctypes.byref(bare), 64) == need                                      # pointers are not looked at
    for bad in (None, ctypes.byref(cache(desc(layers=0))), ctypes.byref(cache(rows=0))):
        assert lib.fbq_cache_evict_workspace_bytes(bad, 64) == 0
    assert lib.fbq_cache_evict_workspace_bytes(ctypes.byref(c), 0) == lib.fbq_cache_evict_workspace_bytes(ctypes.byref(c), (1 << 24) + 1) == 0
    far = OK + (1 << 30)
    go = lambda c=c, w=OK, out=far, stride=512, width=64, keep=OK, first=0, recent=0, info=None, ws=OK, size=1 << 40: \
        lib.fbq_cache_evict(ctypes.byref(c) if c is not None else None, w, out, stride, width, keep, first, recent, info, ws, size, None)
    assert go(c=None) == go(c=cache(refs=None)) == 1
    assert go(width=0) == go(width=(1 << 24) + 1) == go(stride=511) == go(first=-1) == go(recent=-1) == go(first=(1 << 24) + 1) == 2
    assert go(c=cache(desc(layers=4096, kv_heads=1024), rows=65536, max_pages=1), stride=1 << 40) == go(stride=(1 << 48) + 1) == 3
    assert go(out=OK + 512) == go(out=OK - 512) == 3             # one over a part of the other
    assert go(w=None) == go(out=None) == go(keep=None) == go(ws=None) == 1
    assert go(w=ODD2) == go(out=ODD2) == go(keep=ODD2) == go(info=ODD2) == go(ws=ODD8) == 4
    assert go(size=need - 1) == 5


# ------------------------------------------------------------------ the binding

HERE = SimpleNamespace(cuda_stream=0)


@pytest.fixture
def host(monkeypatch):
    """Addresses of host tensors pass, and a call that reaches the library raises."""
    monkeypatch.setattr(kv, "_dev_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(kv, "_stream", lambda stream=None: 0)
    monkeypatch.setattr(kv, "_tokens", lambda cache, t, what, heads=None: (t.data_ptr(), t.stride(0), t.shape[0]))
    real = fbq.load()

    def reached(code, what):
        if what != "Cache":
            raise AssertionError(f"{what} was called")
    stub = SimpleNamespace(fbq_check_cache=real.fbq_check_cache, fbq_cache_evict_workspace_bytes=real.fbq_cache_evict_workspace_bytes)
    for name in ("fbq_cache_read", "fbq_attention_weights", "fbq_cache_evict"):
        setattr(stub, name, lambda *a: 0)
    monkeypatch.setattr(kv.fbq, "load", lambda: stub)
    monkeypatch.setattr(kv, "_check", reached)
    return fbq.cache_create(2, 8, 16, 2, 80, 4, 3, device="cpu", bits=4)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_caches_that_are_none(host):
    t = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype)
    go = lambda pool, **how: fbq.Cache(pool, t(4, 3), t(4), t(8), **how)
    good = t(2, 8, 2, 2, 16, 56, dtype=torch.uint8)
    assert go(good, dtype=torch.bfloat16, dim=80).head_dim == 80 and go(good, dtype=torch.float16, dim=96).head_dim == 96 and host.head_dim == 80 and host.dtype == torch.float16
    for pool, how in ((good, {}), (good, dict(dtype=torch.float16)), (good, dict(dtype=torch.float32, dim=80)), (good, dict(dtype=torch.float16, dim=128)),
                      (good, dict(dtype=torch.float16, dim=300)), (good.to(torch.int8), dict(dtype=torch.float16, dim=80)), (good.half(), dict(dtype=torch.bfloat16)),
                      (good.half(), dict(dim=80))):
        with pytest.raises(ValueError):
            go(pool, **how)
    with pytest.raises(ValueError):
        fbq.cache_create(2, 8, 16, 2, 80, 4, 3, device="cpu", bits=8)
    for name, value in (("dtype", torch.bfloat16), ("dim", 96), ("pool", good)):
        with pytest.raises(AttributeError):
            setattr(host, name, value)
    part = host.rows(1, 3)
    assert part.dim == 80 and part.dtype == torch.float16 and part.table.shape == (2, 3)


def test_read_refuses(host):
    f = lambda *shape: torch.zeros(shape)
    go = lambda tokens=4, start=ints(0, 0, 0, 0), q_start=None, k=None, v=None: fbq.cache_read(host, 0, tokens, start, q_start=q_start, k=f(tokens, 2, 80) if k is None else k,
                                                                                              v=f(tokens, 2, 80) if v is None else v, stream=HERE)
    for bad in (dict(start=ints(0, 0)), dict(start=torch.zeros(4)), dict(q_start=ints(0, 1, 2, 3)), dict(k=f(4, 2, 64)), dict(v=f(3, 2, 80)), dict(k=f(4, 2, 80).half())):
        with pytest.raises(ValueError):
            go(**bad)
    with pytest.raises(AssertionError, match="fbq_cache_read was called"):
        go()


def test_weights_refuse(host):
    w, lse, q = torch.zeros(4, 2, 48), torch.zeros(4, 4), torch.zeros(4, 4, 80, dtype=torch.float16)
    go = lambda weights=w, lse=lse, **how: fbq.attention_weights(host, 0, q, lse, weights, stream=HERE, **how)
    for bad in (dict(weights=None), dict(weights=w[:3]), dict(weights=w[:, :1]), dict(weights=w.double()), dict(weights=w[0]), dict(out=torch.zeros(4, 2, 47)), dict(out=w.half()), dict(lse=None),
                dict(lse=lse[:3]), dict(lse=lse.double())):
        with pytest.raises(ValueError):
            go(**bad)
    for good in ({}, dict(weights=None, out=w), dict(out=torch.zeros(4, 2, 48))):
        with pytest.raises(AssertionError, match="fbq_attention_weights was called"):
            go(**good)


def test_evict_refuses(host):
    w = torch.zeros(2, 6, 2, 48)
    go = lambda weights=w[:, 1:5], keep=ints(1, 1, 1, 1), **how: fbq.cache_evict(host, weights, keep, workspace=torch.empty(1 << 16, dtype=torch.uint8), stream=HERE, **how)
    for bad in (dict(weights=w), dict(weights=w[:1, :4]), dict(weights=w[:, :4].double()), dict(weights=w[:, :4, :, ::2]), dict(keep=ints(1, 1)), dict(keep=torch.zeros(4)),
                dict(out=torch.zeros(2, 4, 2, 48)), dict(out=torch.zeros(2, 4, 2, 47)), dict(info=ints(0))):
        with pytest.raises(ValueError):
            go(**bad)
    for good in ({}, dict(out=torch.zeros(2, 6, 2, 48)[:, :4]), dict(info=ints(0, 0), first=3, recent=2)):
        with pytest.raises(AssertionError, match="fbq_cache_evict was called"):
            go(**good)


def test_kernels_have_their_registers(kernels):  # noqa: F811
    """Two blocks a CU up to 128 features, one beyond: registers and LDS; the few-row kernels, whose loads are waited for by count, without scratch memory."""
    found = {n: k for n, k in kernels.items() if re.search(r"fbq_(attend4_\w+|weigh_\w+|append4|evict_\w+|cache_read)_kernel", n)}
    count = lambda s: len([n for n in found if s in n])
    assert (count("attend4_few"), count("attend4_many"), count("attend4_both"), count("weigh_few"), count("weigh_many"), count("append4"), count("cache_read")) == (10, 10, 6, 20, 20, 20, 4)
    for n, k in found.items():
        if "attend4" in n:
            alone = re.search(r"[68]>", n)
            assert k[".vgpr_count"] <= (512 if alone else 256), n
            assert k[".group_segment_fixed_size"] <= (160 if alone else 80) * 1024, n
        if re.search("few|append4|evict|read", n):
            assert k[".private_segment_fixed_size"] <= 64 and k[".vgpr_spill_count"] == 0, (n, k[".private_segment_fixed_size"])
