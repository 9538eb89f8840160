"""What the binding of the cache refuses before it calls the library (no GPU: host tensors stand in for the device's, and nothing is launched)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2501_16385_amd as fbq
from paper_2501_16385_amd import cache as kv

HERE = SimpleNamespace(cuda_stream=0)


@pytest.fixture
def host(monkeypatch):
    """Addresses of host tensors pass, and a call that reaches the library raises."""
    monkeypatch.setattr(kv, "_dev_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(kv, "_stream", lambda stream=None: 0)

    def reached(code, what):
        if what != "Cache":
            raise AssertionError(f"{what} was called")

    cache = fbq.cache_create(1, 8, 16, 2, 64, 4, 3, device="cpu")
    real = fbq.load()
    stub = SimpleNamespace(fbq_check_cache=real.fbq_check_cache, fbq_cache_workspace_bytes=real.fbq_cache_workspace_bytes)
    for name in ("fbq_cache_reserve", "fbq_cache_fork", "fbq_cache_compact", "fbq_cache_free", "fbq_cache_copy", "fbq_cache_append"):
        setattr(stub, name, lambda *a: 0)
    monkeypatch.setattr(kv.fbq, "load", lambda: stub)
    monkeypatch.setattr(kv, "_check", reached)
    return cache


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def calls(cache, info):
    """(how many numbers info has to take, the call)"""
    ws = torch.empty(1 << 12, dtype=torch.uint8)
    return {"reserve": (1, lambda: fbq.cache_reserve(cache, ints(1, 1, 1, 1), start=ints(0, 0, 0, 0), info=info, stream=HERE)),
            "fork": (2, lambda: fbq.cache_fork(cache, ints(0), ints(1), info=info, workspace=ws, stream=HERE)),
            "compact": (2, lambda: fbq.cache_compact(cache, info=info, workspace=ws, stream=HERE))}


@pytest.mark.parametrize("name", ["reserve", "fork", "compact"])
def test_info_takes_what_is_written_there(host, name):
    need, _ = calls(host, None)[name]
    for short in [ints(*[0] * n) for n in range(need)] + [torch.zeros(2), torch.zeros(2, dtype=torch.int64)]:
        with pytest.raises(ValueError, match="info"):
            calls(host, short)[name][1]()
    for enough in (None, ints(*[0] * need), ints(0, 0, 0)):
        with pytest.raises(AssertionError, match="was called"):
            calls(host, enough)[name][1]()


def test_compact_moves_pages_of_one_pool(host):
    """The new table names pages of the pool that they move in: `out` has to be a cache of that one."""
    ws = torch.empty(1 << 12, dtype=torch.uint8)
    go = lambda out: fbq.cache_compact(host, out=out, workspace=ws, stream=HERE)
    another = lambda pool, table=host.table: fbq.Cache(pool, table.clone(), host.lengths, torch.zeros(pool.shape[1], dtype=torch.int32))
    for wrong in (another(host.pool.clone()), another(host.pool.view(torch.bfloat16)), another(host.pool.view(1, 8, 2, 1, 16, 128)), another(host.pool[:, :4])):
        with pytest.raises(ValueError, match="pool"):
            go(wrong)
    with pytest.raises(ValueError, match="shape"):
        go(another(host.pool, host.table[:, :2]))
    with pytest.raises(AssertionError, match="was called"):
        go(another(host.pool))


def test_compact_is_of_all_rows(host):
    """Pages of rows that are not in the table would move all the same."""
    ws = torch.empty(1 << 12, dtype=torch.uint8)
    for part in (host.rows(0, 3), host.rows(1, 4), host.rows(1, 3).rows(0, 2)):
        with pytest.raises(ValueError, match="all rows"):
            fbq.cache_compact(part, workspace=ws, stream=HERE)
        whole = fbq.Cache(host.pool, part.table.clone(), part.lengths, host.refs.clone())
        with pytest.raises(ValueError, match="all rows"):
            fbq.cache_compact(whole, out=part, workspace=ws, stream=HERE)
    with pytest.raises(AssertionError, match="was called"):
        fbq.cache_compact(host.rows(0, 4), workspace=ws, stream=HERE)


@pytest.mark.parametrize("name", ["pool", "table", "lengths", "refs"])
def test_a_cache_does_not_go_on_with_the_old_one_of_two_tensors(host, name):
    """Calls take the addresses that the Cache was made with: another tensor in a field would be left out of them, silently."""
    old = getattr(host, name)
    with pytest.raises(AttributeError, match=name):
        setattr(host, name, old.clone())
    assert getattr(host, name) is old and old.data_ptr() == getattr(host._c, name)
    getattr(host, name).zero_()
