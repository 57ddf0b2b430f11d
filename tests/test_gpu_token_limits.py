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


def squared_norms(desc, codes, scales, dy, lengths=None):
    need = dp.dp_checkpoint_workspace_bytes(desc)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda:0")
    sq = torch.full((desc.n + 1,), -7.0, device="cuda:0")
    dp.dp_checkpoint_example_grad(desc, codes, scales, dy, None, None, sq, ws, lengths=lengths, ws_bytes=need)
    assert bool((ws[need:] == 0xA5).all()) and float(sq[desc.n]) == -7.0
    return sq[:desc.n].double()


# few tokens of wide layers: norms by Gram matrices, some with features shared between workgroups, of one tile of tokens and of several; and small layers
CANCELLING = [(20, 64, 2048, 2048, 0), (32, 64, 768, 768, 1), (12, 33, 1500, 1501, 1), (24, 16, 2048, 1030, 0), (300, 2, 1792, 576, 1), (6, 200, 2100, 2050, 0),
              (3, 130, 4096, 4096, 1), (64, 32, 64, 64, 0), (700, 10, 520, 300, 1), (40, 33, 2048, 2049, 1), (10, 200, 4096, 4100, 1), (12, 64, 4096, 4096, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CANCELLING, ids=str)
def test_norms_of_gradients_that_cancel(case, dtype):
    """Tokens nearly alike, whose gradients add up to nothing, as a key projection's do: the weight gradient is far smaller than its terms.  Its norm is
    what the contraction makes of it, or a sum over pairs of tokens that has not lost more than a quarter; never below zero and never zero."""
    n, tokens, cin, cout, bias = case
    desc = layer(n, tokens, cin, cout, dtype, bias)
    gen = torch.Generator("cuda:0").manual_seed(n)
    x = torch.randn((n, 1, cin), generator=gen, device="cuda:0") * 4.0
    spread = 2.0 ** -(torch.arange(n, device="cuda:0") % 7 * 2.0)            # from tokens of their own to tokens all alike
    x = x + spread[:, None, None] * torch.randn((n, tokens, cin), generator=gen, device="cuda:0")
    codes, scales, x = checkpoint(x.reshape(n * tokens, cin).to(torch.bfloat16))
    dy = torch.randn((n, tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)
    lengths = torch.full((n,), tokens, dtype=torch.int32, device="cuda:0")
    lengths[n // 2] = 0
    if tokens > 3:
        lengths[n // 3] = tokens // 2 * 2 - 2
    dy[:, 1::2] = -dy[:, 0:tokens // 2 * 2:2]                                # opposite pairs
    if tokens % 2:
        dy[:, -1] = 0.0
    odd = torch.arange(n, device="cuda:0") % 7 == 5                          # and some that do not cancel
    dy[odd] = torch.randn((int(odd.sum()), tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)
    there = torch.arange(tokens, device="cuda:0")[None] < lengths[:, None]
    got = squared_norms(desc, codes, scales, torch.where(there[..., None], dy, math.nan).to(dtype), lengths)
    g, x = dy.double() * there[..., None], x.view(n, tokens, cin)
    planes = 1 if dtype == torch.bfloat16 else 3
    for i in range(n):
        w = g[i].t() @ x[i]
        off = (planes * tokens + 2) * U * (g[i].abs().t() @ x[i].abs())
        b, off_b = g[i].sum(0) * bias, (tokens + 2) * U * g[i].abs().sum(0) * bias
        want = float((w ** 2).sum() + (b ** 2).sum())
        far = float((2 * w.abs() * off + off ** 2).sum() + (2 * b.abs() * off_b + off_b ** 2).sum()) + 256 * U * want
        terms = float(((g[i].abs() @ g[i].abs().t()) * (x[i].abs() @ x[i].abs().t() + bias)).sum())
        gram = min((cin + cout + 256) * U * terms, want / 3)
        assert abs(float(got[i]) - want) <= max(far, gram), (i, float(got[i]), want)
        assert float(got[i]) >= 0.0 and (want <= far or float(got[i]) > 0.0), (i, float(got[i]), want)


def test_norms_that_are_not_numbers_and_their_neighbours():
    """A NaN or infinity in an example's operands: its squared norm is not a number that a factor above 0 comes from; the others are theirs."""
    n, tokens, cin, cout = 20, 64, 2048, 2048
    desc = layer(n, tokens, cin, cout)
    gen = torch.Generator("cuda:0").manual_seed(8)
    x = torch.randn((n * tokens, cin), generator=gen, device="cuda:0").to(torch.bfloat16)
    dy = torch.randn((n, tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)
    clean = squared_norms(desc, *checkpoint(x)[:2], dy)
    x.view(n, tokens, cin)[3, 5, 7] = math.nan
    dy[5, 0, 0] = math.nan
    dy[7, 63, 2047] = math.inf
    dy[9] *= 1e30                                    # squares beyond fp32
    codes, scales, _ = checkpoint(x)
    got = squared_norms(desc, codes, scales, dy)
    factors = torch.empty(n, device="cuda:0")
    dp.dp_clip_factors(got.float(), 1.0, n, factors)
    broken = torch.zeros(n, dtype=torch.bool, device="cuda:0")
    broken[[3, 5, 7, 9]] = True
    assert bool((factors[broken] == 0.0).all())
    assert torch.equal(got[~broken], clean[~broken]) and bool((clean > 0.0).all())


@pytest.mark.parametrize("width,tokens,n", [(64, 32, 64), (2048, 64, 16)])
def test_share_of_an_example_whose_tokens_are_nearly_alike(width, tokens, n):
    """The attention block on such inputs: the key projection's gradient cancels, the block's norm does not lose it, and no example's share of the
    clipped sum passes the bound."""
    block = dp.PrivateAttention(n, tokens, width, heads=4, clip_c=1e-4, sigma=0.0, total_batch=n, device="cuda:0")
    gen = torch.Generator("cuda:0").manual_seed(9)
    x = torch.randn((n, 1, width), generator=gen, device="cuda:0") * 3 + 2.0 ** -6 * torch.randn((n, tokens, width), generator=gen, device="cuda:0")
    block.forward(x.to(torch.bfloat16).contiguous())
    block.backward(torch.randn((n, tokens, width), generator=gen, device="cuda:0").to(torch.bfloat16))
    values = []
    for codes, scales in (block.inputs, block.mixed):
        back = torch.empty((n * tokens, width), dtype=torch.float32, device="cuda:0")
        dp.dp_checkpoint_read(codes, scales, back)
        values.append(back.double().view(n, tokens, width))
    for i in range(n):
        squares = [float(((g[i].double().t() @ values[0 if k < 3 else 1][i]) ** 2).sum()) for k, g in enumerate(block.grads)]
        total = sum(squares) + float((block.g_table[i].double() ** 2).sum())
        f = min(1.0, block.clip_c / math.sqrt(float(block.total_sqnorm[i])))
        assert f * math.sqrt(total) <= block.clip_c * (1.0 + 2.0 ** -9), (i, f * math.sqrt(total))
        for k in range(4):
            assert float(block.sqnorm[k, i]) >= squares[k] * (1.0 - 2.0 ** -8), (i, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_recorded_norms_of_gradients_that_cancel(dtype):
    """Replays with other examples cancelling each time give the eager results."""
    n, tokens, cin, cout = 20, 64, 2048, 2048
    desc = layer(n, tokens, cin, cout, dtype)
    gen = torch.Generator("cuda:0").manual_seed(10)
    codes, scales, _ = checkpoint((torch.randn((n, 1, cin), generator=gen, device="cuda:0") + 2.0 ** -5 * torch.randn((n, tokens, cin), generator=gen, device="cuda:0"))
                                  .reshape(n * tokens, cin).to(torch.bfloat16))
    dy, sq = torch.empty((n, tokens, cout), dtype=dtype, device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(dp.dp_checkpoint_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")

    def fresh(seed):
        gen = torch.Generator("cuda:0").manual_seed(seed)
        dy.copy_(torch.randn(dy.shape, generator=gen, device="cuda:0"))
        some = torch.rand(n, generator=gen, device="cuda:0") < 0.5
        dy[some, 1::2] = -dy[some, 0::2]

    def call():
        dp.dp_checkpoint_example_grad(desc, codes, scales, dy, None, None, sq, ws)
    fresh(0)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(1, 6):
        fresh(seed)
        call()
        torch.cuda.synchronize()
        eager = sq.clone()
        sq.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, sq) and bool((sq > 0.0).all())


@pytest.mark.parametrize("n,tokens", [(5003, 2), (2049, 6), (9000, 1)])
def test_norms_of_many_examples_some_of_which_cancel(n, tokens):
    """More examples than are looked at together."""
    cin, cout = 256, 288
    desc = layer(n, tokens, cin, cout)
    gen = torch.Generator("cuda:0").manual_seed(n)
    spread = 2.0 ** -(torch.arange(n, device="cuda:0") % 5 * 3.0)[:, None, None]
    x = torch.randn((n, 1, cin), generator=gen, device="cuda:0") * 4.0 + spread * torch.randn((n, tokens, cin), generator=gen, device="cuda:0")
    codes, scales, x = checkpoint(x.reshape(n * tokens, cin).to(torch.bfloat16))
    dy = torch.randn((n, tokens, cout), generator=gen, device="cuda:0").to(torch.bfloat16)
    if tokens > 1:
        dy[:, 1::2] = -dy[:, 0::2]
    got = squared_norms(desc, codes, scales, dy)
    for i in range(0, n, 500):
        g, v = dy[i:i + 500].double().transpose(1, 2).contiguous(), x.view(n, tokens, cin)[i:i + 500].contiguous()
        w, off = g @ v, (tokens + 2) * U * (g.abs() @ v.abs())
        want = (w ** 2).sum((1, 2))
        far = (2 * w.abs() * off + off ** 2).sum((1, 2)) + 256 * U * want
        assert bool(((got[i:i + 500] - want).abs() <= torch.maximum(far, want / 3)).all())
        assert torch.equal(got[i:i + 500] > 0.0, want > 0.0)         # (two tokens that round to one and cancel leave nothing)
