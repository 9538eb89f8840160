"""Pages whose chunks, in all layers, are more than one dimension of a grid has blocks."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers,kv_heads,D", [(4096, 32, 128), (4095, 41, 120)])
def test_fork_and_copy(layers, kv_heads, D):
    """4096 layers with a page of 256 KiB each (16 chunks), and 4095 with one of 307 KiB (19 chunks, the last one begun)."""
    import paper_2501_16385_amd as fbq
    cache = fbq.cache_create(layers, 3, 16, kv_heads, D, 2, 2)
    bits = cache.pool.view(torch.int16)
    bits.random_(generator=torch.Generator(device="cuda").manual_seed(1))
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache.table[0, 0], cache.lengths[0], cache.refs[1] = 1, 7, 1
    page, others, info = bits[:, 1].clone(), bits[:, 2].clone(), ints(9, 9)
    fbq.cache_fork(cache, ints(0), ints(1), info=info)
    assert info.tolist() == [0, 0] and cache.table.tolist() == [[1, -1], [0, -1]] and cache.lengths.tolist() == [7, 7] and cache.refs.tolist() == [1, 1, 0]
    assert torch.equal(bits[:, 0], page) and torch.equal(bits[:, 1], page) and torch.equal(bits[:, 2], others)
    fbq.cache_copy(cache, ints(2), ints(0))
    assert torch.equal(bits[:, 0], others) and torch.equal(bits[:, 1], page) and torch.equal(bits[:, 2], others)
