"""The decode loop under a budget until a second row is over it, too: how many rows each step cuts back, and what they hold."""
import pytest
import torch  # noqa: F401

from test_gpu_decode_budget import begun

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
def test_rows_come_to_their_budget_one_after_the_other(bits):
    from paper_2501_16385_amd.decode_loop import Budget
    stack = begun(bits, 2, Budget(24, first=3, recent=6, decay=0.9))          # rows of 33, 10 and 17 tokens
    for step in range(1, 18):
        stack.step()
        n = [min(24, 33 + step), min(24, 10 + step), min(24, 17 + step)]
        assert stack.cache.lengths.tolist() == n
        # 17 + 8 and 10 + 15 are the first beyond 24
        assert stack.evicted.tolist() == [1 + (step >= 8) + (step >= 15), 0] and stack.most_skipped.tolist() == [0]
        for b, tokens in enumerate(n):
            assert (stack.weights[:, b, :, tokens:] == 0).all() and torch.isfinite(stack.weights[:, b]).all()
            held = [p for p in stack.cache.table[b].tolist() if p >= 0]
            assert len(held) == -(-tokens // 16) and all(stack.cache.refs[p] == 1 for p in held)
