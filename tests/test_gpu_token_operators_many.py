"""Calls of more workgroups than a launch has room for (fewer than 2^32 threads): what they make of their first and last rows or examples, against
calls of those by themselves."""
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu


def needs(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of device memory are not free")


@pytest.mark.parametrize("queries", [1, 8])
def test_softmax_of_many_heads(queries):
    """17 million rows of one query each, and eight times as many."""
    needs(8)
    n, heads, keys = 65535, 260, 2
    gen = torch.Generator("cuda:0").manual_seed(queries)
    scores = torch.randn((n, heads, queries, keys), generator=gen, device="cuda:0", dtype=torch.bfloat16)
    dprobs = torch.randn(scores.shape, generator=gen, device="cuda:0", dtype=torch.bfloat16)
    table = torch.randn((2, heads), generator=gen, device="cuda:0")

    def both(first, count):
        desc = dp.BiasDesc(in_dtype=dp.DP_BF16, n=count, heads=heads, queries=queries, keys=keys, buckets=2, max_distance=2, bidirectional=0, causal=0,
                           query_offset=0, scale=1.0)
        s, d = scores[first:first + count], dprobs[first:first + count]
        probs, dscores = torch.full_like(s, 7.0), torch.full_like(s, 7.0)
        g, sq = torch.full((count, 2, heads), 7.0, device="cuda:0"), torch.full((count,), 7.0, device="cuda:0")
        dp.dp_bias_softmax(desc, s, table, probs)
        dp.dp_bias_softmax_backward(desc, probs, d, dscores, g, sq, torch.empty(dp.dp_bias_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0"))
        return probs, dscores, g, sq
    whole = both(0, n)
    # a part may go by another kernel, whose sums of two differ by nothing but whose results are rounded to bf16 from fp32 ones a step apart
    for first, count in ((0, 3000), (n - 3000, 3000), (n // 2, 500)):
        for got, want in zip((t[first:first + count] for t in whole), both(first, count)):
            off = (got.double() - want.double()).abs()
            assert bool((off <= (2.0 ** -7 if want.dtype == torch.bfloat16 else 2.0 ** -6) * want.double().abs() + 2.0 ** -7).all())
    for t in whole[:2]:
        assert bool((t != 7.0).all())
    assert bool(((whole[0].float().sum(-1) - 1.0).abs() <= 2.0 ** -7).all())


def test_checkpoint_of_many_values():
    """2^35 values of fp32, written and read."""
    needs(175)
    rows, features = (1 << 25) + 1000, 1024
    x = torch.empty((rows, features), device="cuda:0").fill_(0.75)
    last = torch.randn((500, features), generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0")
    x[-500:] = last
    codes = torch.empty((rows, features), dtype=torch.uint8, device="cuda:0")
    scales = torch.empty((rows, features // 32), dtype=torch.uint8, device="cuda:0")
    dp.dp_checkpoint_write(x, codes, scales)
    alone = torch.empty((500, features), dtype=torch.uint8, device="cuda:0"), torch.empty((500, features // 32), dtype=torch.uint8, device="cuda:0")
    dp.dp_checkpoint_write(last, *alone)
    assert torch.equal(codes[-500:], alone[0]) and torch.equal(scales[-500:], alone[1])
    first = codes[0].clone()
    for part in codes[:-500].split(1 << 22):
        assert bool((part == first).all())
    x.fill_(9.0)
    dp.dp_checkpoint_read(codes, scales, x)
    want = torch.empty_like(last)
    dp.dp_checkpoint_read(*alone, want)
    assert torch.equal(x[-500:], want)
    for part in x[:-500].split(1 << 22):
        assert bool((part == 0.75).all())


@pytest.mark.parametrize("ragged", [False, True])
def test_stored_gradients_of_many_tiles(ragged):
    """65535 examples of 512 tiles each, those of the bias among them."""
    needs(40)
    n, cin, cout = 65535, 1, 32768
    desc = dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dp.DP_BF16, n=n, cin=cin, cout=cout, h=1, w=1, has_bias=1)
    gen = torch.Generator("cuda:0").manual_seed(3)
    x = torch.randn((n, cin), generator=gen, device="cuda:0").to(torch.bfloat16)
    codes, scales = torch.empty((n, 32), dtype=torch.uint8, device="cuda:0"), torch.empty((n, 1), dtype=torch.uint8, device="cuda:0")
    dp.dp_checkpoint_write(x, codes, scales)
    values = torch.empty((n, cin), device="cuda:0")
    dp.dp_checkpoint_read(codes, scales, values)
    dy = torch.randn((n, cout), generator=gen, device="cuda:0", dtype=torch.bfloat16)
    lengths = torch.randint(0, 2, (n,), generator=gen, device="cuda:0", dtype=torch.int32) if ragged else None
    g_w, g_b = torch.full((n, cout), 7.0, device="cuda:0"), torch.full((n, cout), 7.0, device="cuda:0")
    sq = torch.full((n,), 7.0, device="cuda:0")
    ws = torch.empty(dp.dp_checkpoint_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dp.dp_checkpoint_example_grad(desc, codes, scales, dy, g_w, g_b, sq, ws, lengths=lengths)
    for i in range(0, n, 4096):                      # one product each: exact
        part = slice(i, i + 4096)
        there = 1.0 if lengths is None else lengths[part, None].float()
        db = dy[part].float() * there
        assert torch.equal(g_b[part], db) and torch.equal(g_w[part], db * values[part])
        want = (db.double() ** 2).sum(1) * (1.0 + values[part, 0].double() ** 2)
        assert bool(((sq[part].double() - want).abs() <= 600 * 2.0 ** -24 * want).all())
