"""Layer norm and RMS norm of tokens, and their backward pass with per-example gradients, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the results' type
EPS = 1e-5


def depth(features):
    """Additions that a sum over a row goes through: 32 of a thread and 16 of lanes and waves, rows beyond registers as many as a thread has."""
    return 64 + features // 1024


def desc_of(x, **more):
    n, tokens, features = x.shape
    fields = dict(in_dtype=dp.DP_BF16 if x.dtype == torch.bfloat16 else dp.DP_F32, n=n, tokens=tokens, features=features, rms=0, eps=EPS, row_stride=x.stride(1))
    return dp.NormDesc(**{**fields, **more})


def rows(values, dtype, gap=0, skip=0, guard=7.0):
    """[n, tokens, features] rows of a tensor that is `gap` wider, from element `skip` of it on; the tensor around them as well."""
    n, tokens, features = values.shape
    flat = torch.full((n * tokens * (features + gap) + skip + 64,), guard, dtype=dtype, device="cuda:0")
    view = flat[skip:skip + n * tokens * (features + gap)].view(n, tokens, features + gap)[..., :features]
    view.copy_(values)
    return view, flat


def there_of(lengths, n, tokens):
    if lengths is None:
        return torch.ones((n, tokens), dtype=torch.bool, device="cuda:0")
    return torch.arange(tokens, device="cuda:0")[None] < lengths[:, None]


def definition(x, gamma, beta, there, rms, dy=None):
    """y, or dx, g_w, g_b, sqnorm, in 64 bits, each with how far a result may be off."""
    D = depth(x.shape[2])
    x = torch.where(there[..., None], x.double(), 0.0)
    dev = x if rms else x - x.mean(2, keepdim=True)
    r = 1.0 / ((dev ** 2).mean(2, keepdim=True) + EPS).sqrt()
    xhat = dev * r
    off_xhat = 4 * D * U * (1.0 + xhat.abs()) + (0.0 if rms else 8 * U * U * D * D * r * x.abs().amax(2, keepdim=True))
    gamma = torch.ones(x.shape[2], device="cuda:0") if gamma is None else gamma
    g64 = gamma.double()
    if dy is None:
        y = xhat * g64 + (0.0 if beta is None else beta.double())
        y = torch.where(there[..., None], y, 0.0)
        return y, off_xhat * g64.abs() + 2 * U * (y.abs() + (0.0 if beta is None else beta.double().abs()))
    dy = torch.where(there[..., None], dy.double(), 0.0)
    a = dy * g64
    along = (a * xhat).mean(2, keepdim=True)
    level = torch.zeros_like(along) if rms else a.mean(2, keepdim=True)
    dx = r * (a - level - xhat * along)
    mean_abs, mean_along = a.abs().mean(2, keepdim=True), (a * xhat).abs().mean(2, keepdim=True) + a.abs().mean(2, keepdim=True)
    off_dx = 4 * D * U * r * (a.abs() + mean_abs + xhat.abs() * mean_along) + r * (off_xhat * along.abs() + xhat.abs() * (off_xhat * a.abs()).mean(2, keepdim=True))
    g_w, g_b = (dy * xhat).sum(1), dy.sum(1)
    off_w = (dy.abs() * off_xhat).sum(1) + (x.shape[1] + 32) * U * (dy * xhat).abs().sum(1)
    off_b = (x.shape[1] + 32) * U * dy.abs().sum(1)
    return (dx, off_dx), (g_w, off_w), (g_b, off_b)


def close(got, want, off, what):
    far = (got.double() - want).abs() - off - HALF[got.dtype] * (want.abs() + off) - 1e-37
    assert bool((far <= 0.0).all()), (what, float(far.max()), float((got.double() - want).abs().max()))


def check_forward(values, dtype, gamma, beta, lengths=None, rms=0, gap=0, skip=0, in_place=False):
    x, _ = rows(values, dtype, gap, skip)
    y, around = rows(torch.full_like(values, 3.0), dtype, gap, skip)
    there = there_of(lengths, *values.shape[:2])
    want, off = definition(x, gamma, beta, there, rms)
    if in_place:
        y.copy_(x)
        dp.dp_layer_norm(desc_of(y, rms=rms), y, gamma, beta, y, lengths=lengths)
    else:
        dp.dp_layer_norm(desc_of(x, rms=rms), x, gamma, beta, y, lengths=lengths)
    close(y, want, off, ("y", tuple(values.shape), dtype, rms))
    assert bool((y[~there] == 0.0).all())
    y.fill_(7.0)
    assert bool((around == 7.0).all())               # what lies between and behind the rows


def check_backward(values, grads, dtype, gamma, lengths=None, rms=0, gap=0, skip=0, shift=True, in_place=None, stored=True):
    x, _ = rows(values, dtype, gap, skip)
    dy, _ = rows(grads, dtype, gap, skip)
    n, tokens, features = values.shape
    there = there_of(lengths, n, tokens)
    (dx, off_dx), (g_w, off_w), (g_b, off_b) = definition(x, gamma, None, there, rms, dy)
    desc = desc_of(x, rms=rms)
    need = dp.dp_layer_norm_workspace_bytes(desc)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda:0")
    stride = (features + 3) // 4 * 4 + 8
    got_w, got_b = (torch.full((n, stride), 7.0, device="cuda:0") for _ in range(2))
    sq = torch.full((n + 1,), -7.0, device="cuda:0")
    out, around = (x, None) if in_place == "x" else (dy, None) if in_place == "dy" else rows(torch.full_like(values, 3.0), dtype, gap, skip)
    dp.dp_layer_norm_backward(desc, x, gamma, dy, out, got_w if stored else None, got_b if stored and shift else None, sq if stored else None, ws, lengths=lengths,
                              g_stride=stride, ws_bytes=need)
    case = (tuple(values.shape), dtype, rms, gap, skip)
    close(out, dx, off_dx, ("dx",) + case)
    assert bool((out[~there] == 0.0).all()) and bool((ws[need:] == 0xA5).all())
    if around is not None:
        out.fill_(7.0)
        assert bool((around == 7.0).all())
    if not stored:
        return
    close(got_w[:, :features], g_w, off_w, ("g_w",) + case)
    squares, off_sq = g_w ** 2, 2 * g_w.abs() * off_w + off_w ** 2
    if shift:
        close(got_b[:, :features], g_b, off_b, ("g_b",) + case)
        squares, off_sq = squares + g_b ** 2, off_sq + 2 * g_b.abs() * off_b + off_b ** 2
    else:
        assert bool((got_b == 7.0).all())
    assert bool((got_w[:, features:] == 7.0).all()) and bool((got_b[:, features:] == 7.0).all())
    want = squares.sum(1)
    assert bool(((sq[:n].double() - want).abs() <= off_sq.sum(1) + (80 + features / 16) * U * want + 1e-37).all())
    assert float(sq[n]) == -7.0


def data(n, tokens, features, seed, grads=True):
    gen = torch.Generator("cuda:0").manual_seed(seed)
    x = torch.randn((n, tokens, features), generator=gen, device="cuda:0") * torch.exp(torch.randn((n, tokens, 1), generator=gen, device="cuda:0"))
    x += torch.randn((n, tokens, 1), generator=gen, device="cuda:0")
    dy = torch.randn((n, tokens, features), generator=gen, device="cuda:0")
    return x, dy, torch.randn(features, generator=gen, device="cuda:0") * 0.3 + 1.0, torch.randn(features, generator=gen, device="cuda:0") * 0.2


# every kernel, just within and just beyond what a row's threads hold
WIDTHS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1003, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4100, 5000, 8191, 8192, 8193,
          12001, 16383, 16384, 16385, 20000, 33000]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", WIDTHS)
def test_widths(features, dtype):
    for i, (n, tokens) in enumerate(((1, 1), (3, 5), (2, 70))):
        x, dy, gamma, beta = data(n, tokens, features, features + i)
        lengths = torch.tensor([tokens, 0, 3][:n], dtype=torch.int32, device="cuda:0") if i == 1 else None
        for rms in (0, 1):
            check_forward(x, dtype, gamma, beta, lengths, rms)
            check_backward(x, dy, dtype, gamma, lengths, rms)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features,gap,skip", [(40, 3, 1), (41, 0, 1), (41, 1, 0), (300, 5, 0), (1003, 14, 0), (1003, 13, 0), (1003, 14, 1), (2000, 1, 0), (5001, 0, 3),
                                               (16001, 2, 1), (17001, 1, 1)], ids=str)
def test_rows_that_begin_anywhere(features, gap, skip, dtype):
    x, dy, gamma, beta = data(3, 11, features, features + gap)
    lengths = torch.tensor([11, 4, 0], dtype=torch.int32, device="cuda:0")
    for in_place in (False, True):
        check_forward(x, dtype, gamma, beta, lengths, 0, gap, skip, in_place)
    check_forward(x, dtype, None, None, None, 1, gap, skip)
    check_backward(x, dy, dtype, gamma, lengths, 0, gap, skip)
    check_backward(x, dy, dtype, None, None, 1, gap, skip, shift=False)
    for in_place in ("x", "dy"):
        check_backward(x, dy, dtype, gamma, lengths, 0, gap, skip, in_place=in_place)
    check_backward(x, dy, dtype, gamma, lengths, 1, gap, skip, stored=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,tokens,features", [(300, 3, 64), (300, 9, 100), (1000, 1, 768), (2, 3000, 200), (1, 9000, 48), (40, 260, 1500), (1, 700, 5000)], ids=str)
def test_many_tokens_and_many_examples(n, tokens, features, dtype):
    """Workgroups of several rows, several workgroups an example, joins by one workgroup an example and by several."""
    x, dy, gamma, beta = data(n, tokens, features, n)
    lengths = torch.randint(-2, tokens + 3, (n,), device="cuda:0", dtype=torch.int32, generator=torch.Generator("cuda:0").manual_seed(1))
    check_forward(x, dtype, gamma, beta, lengths)
    check_backward(x, dy, dtype, gamma, lengths)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,features", [(300, 48), (300, 700), (300, 1500), (300, 5000), (40, 9000), (70, 18000)], ids=str)
def test_lengths_may_be_any_numbers(tokens, features, dtype):
    """Far below zero and far beyond the tokens: taken as none and all, by every workgroup of an example."""
    x, dy, gamma, beta = data(6, tokens, features, tokens)
    lengths = torch.tensor([-2 ** 31, 2 ** 31 - 1, -2 ** 31 + 5, tokens + 1, -1, 17], dtype=torch.int32, device="cuda:0")
    check_forward(x, dtype, gamma, beta, lengths)
    check_backward(x, dy, dtype, gamma, lengths)


def test_gradients_of_the_tokens_alone():
    """dx not wanted: gradients of scale and shift as with it."""
    x, dy, gamma, _ = data(4, 33, 500, 1)
    for features in (500, 17000):
        x, dy, gamma, _ = data(4, 33, features, 1)
        desc = desc_of(x)
        ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
        results = []
        for dx in (torch.empty_like(x), None):
            g_w, g_b, sq = torch.empty((4, features), device="cuda:0"), torch.empty((4, features), device="cuda:0"), torch.empty(4, device="cuda:0")
            dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, sq, ws)
            results.append((g_w, g_b, sq))
        assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("features", [64, 768, 3001, 20000])
def test_rows_far_from_zero(features):
    """A mean of a thousand deviations, rows of one value, rows of zeros, tiny and large rows."""
    x, dy, gamma, beta = data(2, 6, features, 3)
    x = torch.randn((2, 6, features), generator=torch.Generator("cuda:0").manual_seed(9), device="cuda:0")
    x[:, 0] += 1000.0
    x[:, 1] = 777.7
    x[:, 2] = 0.0
    x[:, 3] *= 1e-6
    x[:, 4] *= 1e12
    for rms in (0, 1):
        check_forward(x, torch.float32, gamma, beta, None, rms)
        check_backward(x, dy, torch.float32, gamma, None, rms)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", [48, 200, 700, 1500, 6000, 18000])
def test_what_lies_beyond_the_lengths_is_not_used(features, dtype):
    n, tokens = 5, 13
    x, dy, gamma, beta = data(n, tokens, features, 5)
    lengths = torch.tensor([13, 0, 1, 12, 5], dtype=torch.int32, device="cuda:0")
    there = there_of(lengths, n, tokens)
    broken = torch.where(torch.arange(tokens, device="cuda:0")[None, :, None] % 2 == 0, math.nan, math.inf)
    check_forward(torch.where(there[..., None], x, broken), dtype, gamma, beta, lengths)
    check_backward(torch.where(there[..., None], x, broken), torch.where(there[..., None], dy, -broken), dtype, gamma, lengths)


@pytest.mark.parametrize("features", [48, 200, 700, 1500, 6000, 18000])
def test_broken_rows_break_their_own_example_only(features):
    n, tokens = 4, 9
    x, dy, gamma, beta = data(n, tokens, features, 6)
    clean = torch.empty_like(x)
    desc = desc_of(x)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")

    def backward():
        dx, g_w, g_b, sq = torch.empty_like(x), torch.empty((n, features), device="cuda:0"), torch.empty((n, features), device="cuda:0"), torch.empty(n, device="cuda:0")
        dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, sq, ws)
        return dx, g_w, g_b, sq
    dp.dp_layer_norm(desc, x, gamma, beta, clean)
    before = backward()
    x[1, 3, features // 2] = math.nan
    x[1, 4, 0] = math.inf
    dy[2, 8, features - 1] = math.nan
    y = torch.empty_like(x)
    dp.dp_layer_norm(desc, x, gamma, beta, y)
    assert bool(y[1, 3:5].isnan().all())
    y[1, 3:5] = clean[1, 3:5]
    assert torch.equal(y, clean)
    after = backward()
    factors = torch.empty(n, device="cuda:0")
    dp.dp_clip_factors(after[3], 1.0, n, factors)
    assert factors[1] == 0.0 and factors[2] == 0.0 and float(factors[0]) > 0.0
    for a, b in zip(before, after):
        assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3])
    assert bool(after[0][1, 3:5].isnan().all()) and bool(after[0][2, 8].isnan().any())
    assert torch.equal(before[0][1, :3], after[0][1, :3]) and torch.equal(before[0][2, :8], after[0][2, :8])


@pytest.mark.parametrize("rms", [0, 1])
def test_gradient_against_differences(rms):
    """Of the sum of y * dy, along random directions, in fp32 against 64-bit differences of the definition."""
    n, tokens, features = 2, 4, 96
    x, dy, gamma, beta = data(n, tokens, features, 8)
    desc = desc_of(x, rms=rms)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dx, g_w, g_b = torch.empty_like(x), torch.empty((n, features), device="cuda:0"), torch.empty((n, features), device="cuda:0")
    dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, None, ws)

    def value(x, gamma, beta):
        dev = x if rms else x - x.mean(2, keepdim=True)
        return ((dev / ((dev ** 2).mean(2, keepdim=True) + EPS).sqrt() * gamma + beta) * dy.double()).sum((1, 2))
    gen = torch.Generator("cuda:0").manual_seed(2)
    for which, grad in enumerate((dx, g_w, g_b)):
        args = [x.double(), gamma.double(), beta.double()]
        step = torch.randn(args[which].shape, generator=gen, device="cuda:0", dtype=torch.float64)
        h = 1e-5
        ends = [value(*[a + s * h * step if i == which else a for i, a in enumerate(args)]) for s in (1.0, -1.0)]
        slope = (ends[0] - ends[1]) / (2 * h)
        along = (grad.double() * step).flatten(1).sum(1)
        # differences are off by h^2 times a third derivative, 1e-10 times numbers of order 10^2, gradients by 2^-24 of a thousand terms
        assert bool(((along - slope).abs() <= 1e-4 * (1.0 + slope.abs())).all())


def test_recorded_and_on_another_stream():
    """Replays on new inputs, with eager calls between them, and two recorded calls that use one workspace in turn."""
    n, tokens, features = 5, 77, 900
    x, dy, gamma, beta = data(n, tokens, features, 4)
    x, dy = x.to(torch.bfloat16), dy.to(torch.bfloat16)
    desc = desc_of(x)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    y, dx, g_w, g_b, sq = torch.empty_like(x), torch.empty_like(x), *(torch.empty((n, features), device="cuda:0") for _ in range(2)), torch.empty(n, device="cuda:0")

    def call(stream=None):
        dp.dp_layer_norm(desc, x, gamma, beta, y, stream=stream)
        dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, sq, ws, stream=stream)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (y, dx, g_w, g_b, sq)]
    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            call()
    side = torch.cuda.Stream()
    for seed in range(4):
        new = data(n, tokens, features, 100 + seed)
        x.copy_(new[0])
        dy.copy_(new[1])
        call()
        eager = results()
        for graph in graphs:
            for t in (y, dx, g_w, g_b, sq):
                t.zero_()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(eager, results()))
        for t in (y, dx, g_w, g_b, sq):
            t.zero_()
        torch.cuda.synchronize()
        call(side)
        assert all(torch.equal(a, b) for a, b in zip(eager, results()))


def test_gradients_go_on_to_the_clipped_sum():
    """g_w and g_b as columns of one matrix, and dp_clip_accumulate of both at once."""
    n, tokens, features = 6, 20, 100
    x, dy, gamma, _ = data(n, tokens, features, 11)
    desc = desc_of(x)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    g, sq, acc = torch.empty((n, 200), device="cuda:0"), torch.empty(n, device="cuda:0"), torch.zeros(200, device="cuda:0")
    dp.dp_layer_norm_backward(desc, x, gamma, dy, None, g, g[:, 100:], sq, ws, g_stride=200)
    dp.dp_clip_accumulate(g, sq, 3.0, n, 200, acc, 200)
    _, (g_w, off_w), (g_b, off_b) = definition(x, gamma, None, there_of(None, n, tokens), 0, dy)
    f = (3.0 / ((g_w ** 2).sum(1) + (g_b ** 2).sum(1)).sqrt()).clamp(max=1.0)[:, None]
    assert float(f.min()) < 1.0
    want, off = torch.cat(((f * g_w).sum(0), (f * g_b).sum(0))), torch.cat(((f * off_w).sum(0), (f * off_b).sum(0)))
    # and the factor: half of the squared norm's error, a square root, a division
    off += 200 * U * torch.cat(((f * g_w).abs().sum(0), (f * g_b).abs().sum(0)))
    close(acc, want, off, "clipped sum")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", [40, 100, 200, 500, 1000, 3001, 9000, 20000])
def test_rows_of_one_value(features, dtype):
    """Whatever the value: no deviation, y is beta and the scale's gradient zero.  A sum of equal values is off by 2^-18 of it at most, and so is its mean, whose
    deviations are taken three times more: 2^-72 of 2^60, far below eps."""
    x = torch.tensor([1e-30, 1.0, -777.7, 1e12, 1e18, 3e-8], device="cuda:0")[None, :, None].expand(2, 6, features).contiguous()
    _, dy, gamma, beta = data(2, 6, features, 1)
    x, dy = x.to(dtype), dy.to(dtype)
    desc = desc_of(x)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    y, dx, g_w, g_b = torch.empty_like(x), torch.empty_like(x), torch.empty((2, features), device="cuda:0"), torch.empty((2, features), device="cuda:0")
    dp.dp_layer_norm(desc, x, gamma, beta, y)
    assert bool(((y.double() - beta.double()).abs() <= HALF[dtype] * beta.double().abs() + 1e-4 * gamma.double().abs()).all())
    if features % 4 == 0:
        dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, None, ws)
        a = dy.double() * gamma.double()
        want = (a - a.mean(2, keepdim=True)) / EPS ** 0.5
        assert bool(((dx.double() - want).abs() <= HALF[dtype] * want.abs() + 1e-3 * (1.0 + a.abs().amax(2, keepdim=True)) / EPS ** 0.5).all())
        assert bool((g_w.double().abs() <= 1e-4 * dy.double().abs().sum(1)).all())


@pytest.mark.parametrize("rms", [0, 1])
@pytest.mark.parametrize("features", [40, 200, 700, 1500, 6000, 18000])
def test_rows_beyond_the_range_are_no_numbers(features, rms):
    """An infinity or a NaN anywhere, or squares whose sum is beyond fp32: nothing of the row passes for a number, nor its example's norm."""
    x, dy, gamma, beta = data(3, 3, features, 2)
    x[0, 0, 7], x[0, 1, features - 1] = math.inf, math.nan
    x[1, 2] *= 1e25
    desc = desc_of(x, rms=rms)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    y, dx, g_w, g_b, sq = torch.empty_like(x), torch.empty_like(x), torch.empty((3, features), device="cuda:0"), torch.empty((3, features), device="cuda:0"), torch.empty(3, device="cuda:0")
    dp.dp_layer_norm(desc, x, gamma, beta, y)
    dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, sq, ws)
    for t in (y, dx):
        bad = t.isnan().all(2)
        assert bad.tolist() == [[True, True, False], [False, False, True], [False, False, False]]
        assert bool(t[~bad].isfinite().all())
    assert sq.isnan().tolist() == [True, True, False]


@pytest.mark.parametrize("features,tokens,stride", [(1000, 1100, 1 << 22), (1001, 1100, (1 << 22) + 1), (4096, 1100000, 4096), (20000, 230000, 20000)], ids=str)
def test_offsets_beyond_2_to_the_32(features, tokens, stride):
    """The last tokens of tensors of 4.5 billion places against the same tokens by themselves: rows far apart, and many of them."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 32 * 2 ** 30:
        pytest.skip("32 GiB of device memory are not free")
    last = 64
    values, grads, gamma, beta = data(1, last, features, 3)
    buffers = [torch.zeros(tokens * stride, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    x, dy = (torch.as_strided(b, (1, tokens, features), (tokens * stride, stride, 1)) for b in buffers)
    x[:, -last:], dy[:, -last:] = values, grads

    def run(x, dy):
        desc = desc_of(x)
        ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
        n, tokens, features = x.shape
        wide = (features + 3) // 4 * 4
        g_w, g_b, sq = torch.empty((1, wide), device="cuda:0"), torch.empty((1, wide), device="cuda:0"), torch.empty(1, device="cuda:0")
        dp.dp_layer_norm_backward(desc, x, gamma, dy, dy, g_w, g_b, sq, ws, g_stride=wide)
        dp.dp_layer_norm(desc, x, gamma, beta, x)
        return x[:, -last:].clone(), dy[:, -last:].clone(), g_w[:, :features], g_b[:, :features], sq
    alone = run(x[:, -last:].clone(), dy[:, -last:].clone())
    whole = run(x, dy)
    for a, b in zip(whole[:2], alone[:2]):
        assert bool(((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 2.0 ** -9).all())      # (held by other numbers of threads)
    # the tokens before them are zeros, with gradients of zeros: the sums are the same numbers in another order
    for a, b in zip(whole[2:], alone[2:]):
        assert bool(((a - b).abs() <= 200 * U * last * b.abs().amax()).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", [41, 129, 300, 513, 1025, 1500, 2047, 3001, 6001, 12001, 17001])
def test_gradients_of_rows_of_one_value(features, dtype):
    """Widths of every backward kernel, no multiples of four among them, packed gradients: bounds as of test_rows_of_one_value."""
    x = torch.tensor([1e-30, 1.0, -777.7, 1e12, 1e18, 3e-8], device="cuda:0")[None, :, None].expand(2, 6, features).contiguous().to(dtype)
    _, dy, gamma, _ = data(2, 6, features, 1)
    dy = dy.to(dtype)
    desc = desc_of(x)
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dx, g_w, g_b = torch.empty_like(x), torch.empty((2, features), device="cuda:0"), torch.empty((2, features), device="cuda:0")
    dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, g_w, g_b, None, ws)
    a = dy.double() * gamma.double()
    want = (a - a.mean(2, keepdim=True)) / EPS ** 0.5
    assert bool(((dx.double() - want).abs() <= HALF[dtype] * want.abs() + 1e-3 * (1.0 + a.abs().amax(2, keepdim=True)) / EPS ** 0.5).all())
    assert bool((g_w.double().abs() <= 1e-4 * dy.double().abs().sum(1)).all())
    close(g_b, dy.double().sum(1), (x.shape[1] + 32) * U * dy.double().abs().sum(1), "g_b")
