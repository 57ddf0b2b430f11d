"""Tensors whose offsets pass 2^32 bytes (and elements): what the token operators make of the last rows, against the same rows by themselves."""
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu


def needs(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB of device memory are not free")


def checkpoint(x):
    rows, features = x.numel() // x.shape[-1], x.shape[-1]
    pitch = dp.dp_checkpoint_pitch(features)
    codes = torch.empty((rows, pitch), dtype=torch.uint8, device="cuda:0")
    scales = torch.empty((rows, pitch // 32), dtype=torch.uint8, device="cuda:0")
    dp.dp_checkpoint_write(x, codes, scales)
    return codes, scales


def test_checkpoint_rows_beyond_four_gib():
    needs(24)
    rows, features = 4_200_000, 1030                  # 8.7 GB of bf16, 4.4 GB of codes
    x = torch.empty((rows, features), dtype=torch.bfloat16, device="cuda:0").fill_(0.75)
    last = torch.randn((500, features), generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0").to(torch.bfloat16)
    x[-500:] = last
    codes, scales = checkpoint(x)
    alone = checkpoint(last)
    assert torch.equal(codes[-500:], alone[0]) and torch.equal(scales[-500:], alone[1])
    first = checkpoint(x[:1])                          # every other row is like the first
    for part in codes[:-500].split(1 << 20):
        assert bool((part == first[0]).all())
    assert bool((scales[:-500] == first[1]).all())
    x.fill_(9.0)
    dp.dp_checkpoint_read(codes, scales, x)
    want = torch.empty_like(last)
    dp.dp_checkpoint_read(*alone, want)
    assert torch.equal(x[-500:], want) and bool((x[rows // 2] == 0.75).all())


@pytest.mark.parametrize("tokens", [64, 3000])
def test_gradients_of_examples_beyond_four_gib(tokens):
    needs(16)
    cin, cout = 2048, 24
    n = (1 << 32) // (tokens * cin) + 3               # codes of the last examples lie beyond
    gen = torch.Generator("cuda:0").manual_seed(2)
    codes = torch.empty((n, tokens, cin), dtype=torch.uint8, device="cuda:0").fill_(0x38)
    scales = torch.empty((n, tokens, cin // 32), dtype=torch.uint8, device="cuda:0").fill_(127)
    dy = torch.zeros((n, tokens, cout), dtype=torch.bfloat16, device="cuda:0")
    some = checkpoint(torch.randn((2 * tokens, cin), generator=gen, device="cuda:0").to(torch.bfloat16))
    codes[-2:], scales[-2:] = some[0].view(2, tokens, cin), some[1].view(2, tokens, -1)
    dy[-2:] = torch.randn((2, tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)

    def layer(m):
        return dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dp.DP_BF16, n=m, cin=cin, cout=cout, h=tokens, w=1, has_bias=0)

    def room(desc, use):
        return torch.empty(max(dp.dp_checkpoint_workspace_bytes(desc, use), 16), dtype=torch.uint8, device="cuda:0")

    x = torch.empty((2 * tokens, cin), dtype=torch.float32, device="cuda:0")
    dp.dp_checkpoint_read(*some, x)
    x, g = x.double().view(2, tokens, cin).cpu(), dy[-2:].double().cpu()
    want = g.transpose(1, 2) @ x
    terms = g.abs().transpose(1, 2) @ x.abs()
    u = 2.0 ** -24
    sq = torch.full((n,), -1.0, device="cuda:0")
    dp.dp_checkpoint_example_grad(layer(n), codes, scales, dy, None, None, sq, room(layer(n), dp.DP_WS_PER_EXAMPLE_GRAD))
    squares = (want ** 2).sum((1, 2))
    # entries off by the additions of their products (or products of Gram matrices, tokens^2 of them), then sums of the squares
    gram = ((g.abs() @ g.abs().transpose(1, 2)) * (x.abs() @ x.abs().transpose(1, 2))).sum((1, 2))
    off = (tokens + 2) * u * terms
    far = torch.maximum((2 * want.abs() * off + off ** 2).sum((1, 2)) + 256 * u * squares, (cin + cout + 256) * u * gram)
    assert bool(((sq[-2:].double().cpu() - squares).abs() <= far).all()) and bool((sq[:-2] == 0.0).all())
    acc = torch.zeros((cout, cin), device="cuda:0")
    dp.dp_checkpoint_clip_accumulate(layer(n), codes, scales, dy, sq, float("inf"), acc, None, room(layer(n), dp.DP_WS_RECOMPUTE))
    # all others add zeros
    assert bool(((acc.double().cpu() - want.sum(0)).abs() <= (2 * tokens + 70) * u * terms.sum(0)).all())


@pytest.mark.parametrize("keys", [60, 66000])
def test_softmax_rows_beyond_four_gib(keys):
    needs(32)
    queries = 65536 + 40
    n = -(-(1 << 32) // (queries * keys)) if keys < 1000 else 1          # 2^32 scores and more
    scores = torch.zeros((n, 1, queries, keys), dtype=torch.bfloat16, device="cuda:0")
    gen = torch.Generator("cuda:0").manual_seed(3)
    last = torch.randn((1, 1, 24, keys), generator=gen, device="cuda:0").to(torch.bfloat16)
    scores[-1, :, -24:] = last
    table = torch.randn((32, 1), generator=gen, device="cuda:0")
    probs = torch.full_like(scores, 7.0)

    def bias(n, queries, offset):
        return dp.BiasDesc(in_dtype=dp.DP_BF16, n=n, heads=1, queries=queries, keys=keys, buckets=32, max_distance=128, bidirectional=1, causal=0,
                           query_offset=offset, scale=0.5)

    dp.dp_bias_softmax(bias(n, queries, 0), scores, table, probs)
    alone = torch.full_like(last, 7.0)
    dp.dp_bias_softmax(bias(1, 24, queries - 24), last, table, alone)
    # the same row by another kernel (several short rows a wave): results next to each other in bf16 at most, where fp32 sums differ in order
    off = (probs[-1, :, -24:].float() - alone[0].float()).abs()
    assert bool((off <= 2.0 ** -7 * alone[0].float() + 1e-30).all())
    assert bool(((probs[-1, :, -24:].double().sum(-1) - 1.0).abs() <= 2.0 ** -8 + 1e-3).all())
    del scores
    dprobs = torch.zeros_like(probs)
    dprobs[-1, :, -24:] = last
    desc = bias(n, queries, 0)
    dscores = torch.full_like(probs, 7.0)
    g, sq = torch.full((n, 32), 7.0, device="cuda:0"), torch.full((n,), 7.0, device="cuda:0")
    dp.dp_bias_softmax_backward(desc, probs, dprobs, dscores, g, sq, torch.empty(dp.dp_bias_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0"))
    p, d = probs[-1, 0, -24:].double().cpu(), dprobs[-1, 0, -24:].double().cpu()
    dot = (p * d).sum(-1, keepdim=True)
    dz = p * (d - dot)
    off = p * ((keys + 2) * 2.0 ** -24 * (p * d).abs().sum(-1, keepdim=True) + 3 * 2.0 ** -24 * (d - dot).abs())
    got = dscores[-1, 0, -24:].double().cpu()
    assert bool(((got - 0.5 * dz).abs() <= 0.5 * off + 2.0 ** -8 * (0.5 * dz).abs() + 2.0 ** -126).all())
    assert bool((dscores[0, 0, :-24] == 0.0).all()) if n > 1 else bool((dscores[0, 0, :: 997][:-1] == 0.0).all())
    assert bool((g[:-1] == 0.0).all()) and bool((sq[:-1] == 0.0).all()) and float(sq[-1]) >= 0.0
    bucket = torch.tensor([[dp.dp_bias_bucket(desc, q - k) for k in (0, keys - 1)] for q in (queries - 24, queries - 1)])
    if (bucket == bucket[0, 0]).all():                 # all places that are not zeros are in one bucket
        assert abs(float(g[-1].sum()) - float(dz.sum())) <= float(off.sum()) + (keys * 24) * 2.0 ** -24 * float(dz.abs().sum())
