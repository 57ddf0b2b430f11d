"""The token operators at the ends of their ranges: calls that go in several launches, values and masks that leave the ordinary path."""
import math

import numpy as np
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def layer(n, tokens, cin, cout, dtype=torch.bfloat16, bias=0):
    return dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dp.DP_BF16 if dtype == torch.bfloat16 else dp.DP_F32, n=n, cin=cin, cout=cout, h=tokens, w=1,
                        has_bias=bias)


def checkpoint(x):
    """codes, scales, and the values they stand for in 64 bits."""
    rows, features = x.shape
    pitch = dp.dp_checkpoint_pitch(features)
    codes = torch.empty((rows, pitch), dtype=torch.uint8, device="cuda:0")
    scales = torch.empty((rows, pitch // 32), dtype=torch.uint8, device="cuda:0")
    back = torch.empty((rows, features), dtype=torch.float32, device="cuda:0")
    dp.dp_checkpoint_write(x, codes, scales)
    dp.dp_checkpoint_read(codes, scales, back)
    return codes, scales, back.double()


@pytest.mark.parametrize("case", [(1669, 64, 768, 768), (1193, 100, 512, 512), (1256, 128, 384, 384)], ids=str)
def test_clipped_sum_of_more_examples_than_a_launch_stays_in_its_workspace(case):
    """The last launch takes more ranges than the ones before it; 8 MB behind the workspace are left alone."""
    n, tokens, cin, cout = case
    desc = layer(*case)
    gen = torch.Generator("cuda:0").manual_seed(n)
    codes, scales, x = checkpoint(torch.randn((n * tokens, cin), generator=gen, device="cuda:0").to(torch.bfloat16))
    dy = (torch.randn((n * tokens, cout), generator=gen, device="cuda:0") * 0.01).to(torch.bfloat16)
    sq = 10.0 ** (torch.rand((n,), generator=gen, device="cuda:0") * 4 - 2)
    need = dp.dp_checkpoint_workspace_bytes(desc, dp.DP_WS_RECOMPUTE)
    ws = torch.full((need + (8 << 20),), 0xA5, dtype=torch.uint8, device="cuda:0")
    acc = torch.zeros((cout, cin), device="cuda:0")
    dp.dp_checkpoint_clip_accumulate(desc, codes, scales, dy, sq, 0.7, acc, None, ws, ws_bytes=need)
    assert bool((ws[need:] == 0xA5).all())
    f = (0.7 / sq.double().sqrt()).clamp(max=1.0).repeat_interleave(tokens)[:, None]
    g = dy.double() * f
    off = (n * tokens + 2 * n + 8) * U * (g.abs().t() @ x.abs())          # every addition off by half a step, or cut
    assert bool(((acc.double() - g.t() @ x).abs() <= off).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("keys,more", [(8, {}), (64, {}), (64, dict(buckets=8, max_distance=20)), (128, dict(bidirectional=0)), (256, dict(max_distance=4096)),
                                       (256, dict(buckets=64, max_distance=300, bidirectional=0))], ids=str)
def test_table_gradient_of_short_rows_in_whole_numbers(keys, more, dtype):
    """Equal probabilities and gradients that cancel in every row: dz are small whole numbers, and so is every sum of them, in any order.  A sum that is
    lost where lanes meet the same word (a row's neighbouring lanes have seven distances in common) shows as a whole number that is missing."""
    n, heads, queries = 9, 40, 60                    # more than 16384 rows: several to a wave
    fields = dict(in_dtype=dp.DP_BF16 if dtype == torch.bfloat16 else dp.DP_F32, n=n, heads=heads, queries=queries, keys=keys, buckets=32, max_distance=128,
                  bidirectional=1, causal=0, query_offset=keys // 3, scale=1.0)
    desc = dp.BiasDesc(**{**fields, **more})
    rng = np.random.default_rng(keys)
    half = rng.integers(-3, 4, (n, heads, queries, keys // 2))
    dz = rng.permuted(np.concatenate([half, -half], axis=3), axis=3)
    probs = torch.full(dz.shape, 1.0 / keys, dtype=dtype, device="cuda:0")
    dprobs = torch.from_numpy(dz * keys).to(dtype).cuda()
    dscores, g = torch.empty_like(probs), torch.empty((n, desc.buckets, heads), device="cuda:0")
    ws = torch.empty(dp.dp_bias_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dp.dp_bias_softmax_backward(desc, probs, dprobs, dscores, g, None, ws)
    assert np.array_equal(dscores.double().cpu().numpy(), dz)
    bucket = np.array([[dp.dp_bias_bucket(desc, keys // 3 + q - k) for k in range(keys)] for q in range(queries)])
    want = np.stack([(dz * (bucket == b)).sum((2, 3)) for b in range(desc.buckets)], axis=1)
    assert np.array_equal(g.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1, 6, 70, 40), (1, 1, 6, 700, 513), (1, 1, 6, 1500, 900), (1, 1, 6, 3001, 2000), (1, 1, 6, 9000, 8191), (1, 1, 6, 20000, 16500),
                                   (1, 1, 6, 40001, 33000), (30, 14, 40, 61, 40), (30, 14, 40, 120, 101), (30, 14, 40, 256, 9)], ids=str)
def test_broken_scores_break_only_what_counts(shape, dtype):
    """A NaN or an infinity among the keys that count: the row is NaN there and zero at the others, in every kernel; rows beside it are untouched."""
    n, heads, queries, keys, length = shape
    desc = dp.BiasDesc(in_dtype=dp.DP_BF16 if dtype == torch.bfloat16 else dp.DP_F32, n=n, heads=heads, queries=queries, keys=keys, buckets=32,
                       max_distance=128, bidirectional=1, causal=0, query_offset=0, scale=1.0)
    gen = torch.Generator("cuda:0").manual_seed(keys)
    scores = torch.randn((n, heads, queries, keys), generator=gen, device="cuda:0").to(dtype)
    table = torch.randn((32, heads), generator=gen, device="cuda:0")
    key_lengths = torch.full((n,), length, dtype=torch.int32, device="cuda:0")
    clean, probs = torch.empty_like(scores), torch.empty_like(scores)
    dp.dp_bias_softmax(desc, scores, table, clean, key_lengths=key_lengths)
    scores[:, :, 0, 3] = math.nan
    scores[:, :, 2, length - 1] = math.inf
    scores[:, :, 4, :length] = math.inf
    scores[:, :, 5, 0] = -math.inf
    scores[:, :, :, length:] = math.nan
    dp.dp_bias_softmax(desc, scores, table, probs, key_lengths=key_lengths)
    assert bool((probs[..., length:] == 0.0).all())
    for q in (0, 2, 4):
        assert bool(probs[:, :, q, :length].isnan().any(-1).all())
    assert bool(probs[:, :, 0, :length].isnan().all())
    for q in (1, 3):
        assert torch.equal(probs[:, :, q], clean[:, :, q])
    assert bool((probs[:, :, 5, 0] == 0.0).all()) and bool(probs[:, :, 5].isfinite().all())


@pytest.mark.parametrize("bias", [0, 1])
def test_clipped_sum_of_tiny_activations_under_tiny_factors(bias):
    """Scales at the format's lowest, gradients that make up for it, and factors from 1 down to 2^-60: no example adds more than its share.  Each
    example is summed by itself, and all of them together."""
    n, tokens, cin, cout = 12, 40, 96, 64
    gen = torch.Generator("cuda:0").manual_seed(4)
    small = torch.randn((n * tokens, cin), generator=gen, device="cuda:0") * 2.0 ** -97
    small[:, 64:] *= 2.0 ** 40                       # other blocks of a row with ordinary scales
    small[:, :32] *= 2.0 ** -10                      # and codes that are no normal e4m3 numbers
    codes, scales, x = checkpoint(small.to(torch.bfloat16))
    assert int(scales.min()) == 27
    dy = (torch.randn((n * tokens, cout), generator=gen, device="cuda:0") * 2.0 ** 90).to(torch.bfloat16)
    powers = torch.tensor([0, -1, -15, -16, -17, -26, -27, -28, -40, -50, -60, -3], dtype=torch.float64, device="cuda:0")
    sq = (2.0 ** (-2 * powers) * (1.7 ** 2)).float()                       # f = min(1, 1 / sqrt(sq))
    f = (1.0 / sq.double().sqrt()).clamp(max=1.0)

    def run(first, count):
        desc = layer(count, tokens, cin, cout, bias=bias)
        rows = slice(first * tokens, (first + count) * tokens)
        ws = torch.empty(max(dp.dp_checkpoint_workspace_bytes(desc, dp.DP_WS_RECOMPUTE), 16), dtype=torch.uint8, device="cuda:0")
        acc, acc_b = torch.zeros((cout, cin), device="cuda:0"), torch.zeros(cout, device="cuda:0") if bias else None
        dp.dp_checkpoint_clip_accumulate(desc, codes[rows], scales[rows].contiguous(), dy[rows], sq[first:first + count].clone(), 1.0, acc, acc_b, ws)
        g = dy[rows].double() * f[first:first + count].repeat_interleave(tokens)[:, None]
        off = (count * tokens + 2 * count + 8) * U * (g.abs().t() @ x[rows].abs()) + 2.0 ** -126
        assert bool(((acc.double() - g.t() @ x[rows]).abs() <= off).all())
        if bias:
            assert bool(((acc_b.double() - g.sum(0)).abs() <= (count * tokens + 8) * U * g.abs().sum(0)).all())
    for i in range(n):
        run(i, 1)
    run(0, n)


def test_clipped_sum_leaves_out_factors_that_are_no_normal_numbers():
    """Bounds so small that factors leave fp32's normal range beside factors that do not: sums stay finite, and right to fp32's smallest numbers."""
    n, tokens, cin, cout = 4, 32, 64, 64
    gen = torch.Generator("cuda:0").manual_seed(5)
    codes, scales, x = checkpoint(torch.randn((n * tokens, cin), generator=gen, device="cuda:0").to(torch.bfloat16))
    codes.view(n, tokens, cin)[:, :, :8] = 0         # sums that stay zero
    x.view(n, tokens, cin)[:, :, :8] = 0.0
    dy = torch.randn((n * tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)
    sq = torch.tensor([1e-6, 1e30, 1e-6, 1e38], device="cuda:0")
    desc = layer(n, tokens, cin, cout)
    for clip_c in (1e-22, 1e-25, 1e-28):
        ws = torch.empty(max(dp.dp_checkpoint_workspace_bytes(desc, dp.DP_WS_RECOMPUTE), 16), dtype=torch.uint8, device="cuda:0")
        acc = torch.zeros((cout, cin), device="cuda:0")
        dp.dp_checkpoint_clip_accumulate(desc, codes, scales, dy, sq, clip_c, acc, None, ws)
        g = dy.double() * (clip_c / sq.double().sqrt()).repeat_interleave(tokens)[:, None]
        off = (n * tokens + 16) * U * (g.abs().t() @ x.abs()) + tokens * 2.0 ** -118
        assert bool(((acc.double() - g.t() @ x).abs() <= off).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_calls_on_another_stream(dtype):
    """On a stream of their own, with everything that the calls read and overwrite in order before them."""
    n, tokens, cin, cout = 6, 64, 96, 200
    desc = layer(n, tokens, cin, cout, dtype, bias=1)
    gen = torch.Generator("cuda:0").manual_seed(6)
    codes, scales, _ = checkpoint(torch.randn((n * tokens, cin), generator=gen, device="cuda:0").to(torch.bfloat16))
    dy = torch.randn((n * tokens, cout), generator=gen, device="cuda:0").to(dtype)
    lengths = torch.tensor([0, 1, 64, 33, 32, 17], dtype=torch.int32, device="cuda:0")
    room = max(dp.dp_checkpoint_workspace_bytes(desc, use) for use in (dp.DP_WS_PER_EXAMPLE_GRAD, dp.DP_WS_RECOMPUTE))
    results = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        sq, acc, acc_b = torch.full((n,), -7.0, device="cuda:0"), torch.zeros((cout, cin), device="cuda:0"), torch.zeros(cout, device="cuda:0")
        ws = torch.empty(room, dtype=torch.uint8, device="cuda:0")
        torch.cuda.synchronize()
        dp.dp_checkpoint_example_grad(desc, codes, scales, dy, None, None, sq, ws, lengths=lengths, stream=stream)
        dp.dp_checkpoint_clip_accumulate(desc, codes, scales, dy, sq, 0.5, acc, acc_b, ws, lengths=lengths, stream=stream)
        torch.cuda.synchronize()
        results.append((sq, acc, acc_b))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and bool((results[0][0] >= 0.0).all())
