"""Eviction with weights and their results in different rows of one tensor, whose layers lie between each other's."""
import pytest
import torch

from test_gpu_eviction import any_cache, evicted
from cache4_cases import F16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("take,give", [((0, 2), (2, 4)), ((3, 5), (0, 2)), ((1, 3), (3, 5))])
def test_other_rows_of_the_same_tensor(take, give):
    import paper_2501_16385_amd as fbq
    cache, table, values = any_cache(16, [90, 80], 2, 64, 16, F16, layers=3)
    both = torch.rand(3, 5, 2, 96, generator=torch.Generator().manual_seed(1))
    want = evicted(values, table, cache.refs.cpu(), [90, 80], both[:, take[0]:take[1]], [20, 30], 1, 2, 16)
    dev = both.cuda()
    fbq.cache_evict(cache, dev[:, take[0]:take[1]], torch.tensor([20, 30], dtype=torch.int32, device="cuda"), first=1, recent=2, out=dev[:, give[0]:give[1]])
    assert cache.lengths.tolist() == want[3] and torch.equal(torch.nan_to_num(cache.pool.cpu().double(), nan=-9.0), torch.nan_to_num(want[0], nan=-9.0))
    got = dev.cpu()
    for b, n in enumerate((90, 80)):
        assert torch.equal(got[:, give[0] + b, :, :n], want[4][:, b, :, :n]) and torch.equal(got[:, give[0] + b, :, n:], both[:, give[0] + b, :, n:])
    others = [r for r in range(5) if not give[0] <= r < give[1]]
    assert torch.equal(got[:, others], both[:, others])


def test_rows_that_overlap_are_refused():
    import paper_2501_16385_amd as fbq
    cache, _, _ = any_cache(16, [90, 80], 2, 64, 16, F16, layers=3)
    dev, keep = torch.zeros(4, 5, 2, 96, device="cuda"), torch.tensor([20, 30], dtype=torch.int32, device="cuda")
    for w, out in ((dev[:3, 0:2], dev[:3, 1:3]), (dev[:3, 3:5], dev[:3, 2:4]), (dev[:3, 0:2], dev[1:, 0:2]), (dev[1:, 1:3], dev[:3, 2:4])):
        with pytest.raises(fbq.FbqError):
            fbq.cache_evict(cache, w, keep, out=out)
    assert cache.lengths.tolist() == [90, 80]
