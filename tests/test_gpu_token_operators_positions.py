"""Positions near the end of 32 bits: query offsets and queries at their largest together."""
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bidirectional", [0, 1])
def test_probabilities_of_the_last_positions(bidirectional):
    """2^30 - 1 queries from position 2^30 on: all keys are in the far bucket, and equal scores are equal probabilities up to the last row."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 32 * 2 ** 30:
        pytest.skip("32 GiB of device memory are not free")
    queries, keys = (1 << 30) - 1, 10
    desc = dp.BiasDesc(in_dtype=dp.DP_BF16, n=1, heads=1, queries=queries, keys=keys, buckets=32, max_distance=4096, bidirectional=bidirectional, causal=0,
                       query_offset=1 << 30, scale=1.0)
    table = torch.randn((32, 1), generator=torch.Generator().manual_seed(0)).cuda() * 4
    rows = torch.zeros((queries, keys), dtype=torch.bfloat16, device="cuda:0")
    dp.dp_bias_softmax(desc, rows, table, rows)
    tenth = torch.tensor(0.1, dtype=torch.bfloat16)
    for part in (rows[-(1 << 16):], rows[:1 << 16], rows[:: 1 << 14]):
        assert bool((part == tenth.cuda()).all())
