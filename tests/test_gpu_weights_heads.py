"""Attention weights of more than 16 query rows a head for every padded head size, heads that fill it and heads that do not, over caches of 16 and of 4 bits, against 64 bits."""
import pytest

from cache4_cases import BF16, F16
from test_gpu_eviction import check_weights

import torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 40, 64, 72, 80, 96, 120, 128, 136, 192, 200, 248, 256])
def test_weights_of_prompts(D, dtype, bits):
    check_weights(bits, [150, 64, 1, 90], [150, 30, 1, 17], 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("D,page,heads,kv_heads", [(40, 32, 3, 1), (72, 64, 8, 8), (136, 16, 5, 1), (200, 128, 6, 2), (256, 256, 4, 4)])
def test_weights_of_a_part_of_the_row(D, page, heads, kv_heads, bits):
    """Tokens behind others that are held, tiles that end inside a token, a width that ends inside 64 keys, queries in rows of a fused projection, another layer."""
    check_weights(bits, [400, 130, 77], [33, 20, 0], heads, kv_heads, D, page, F16, seed=D, decay=0.5, width=333, layer=1, layers=2, fused=2)
    check_weights(bits, [400, 130, 77], [33, 20, 0], heads, kv_heads, D, page, BF16, seed=D, scale=-0.1, apart=True)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("D", [192, 256])
def test_weights_of_many_keys_and_tokens(D, bits):
    """Enough keys that two waves, or one, and not four, share 64 of them."""
    check_weights(bits, [128, 100, 61] + [20 + b for b in range(30)], [40, 33, 17] + [2] * 30, 128, 32, D, 16, F16, seed=D, decay=0.25)
