"""Log probabilities of tokens, entropies, alternatives and their gradient, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the results' type
INF = math.inf


def desc_of(x, **more):
    n, tokens, vocab = x.shape
    fields = dict(in_dtype=dp.DP_BF16 if x.dtype == torch.bfloat16 else dp.DP_F32, n=n, tokens=tokens, vocab=vocab, top=0, scale=1.0, row_stride=x.stride(1))
    return dp.LogprobDesc(**{**fields, **more})


def rows(values, dtype, gap=0, skip=0, guard=7.0):
    """[n, tokens, vocab] rows of a tensor that is `gap` wider, from element `skip` of it on; the tensor around them as well."""
    n, tokens, vocab = values.shape
    flat = torch.full((n * tokens * (vocab + gap) + skip + 64,), guard, dtype=dtype, device="cuda:0")
    view = flat[skip:skip + n * tokens * (vocab + gap)].view(n, tokens, vocab + gap)[..., :vocab]
    view.copy_(values)
    return view, flat


def there_of(lengths, n, tokens):
    if lengths is None:
        return torch.ones((n, tokens), dtype=torch.bool, device="cuda:0")
    return torch.arange(tokens, device="cuda:0")[None] < lengths[:, None]


class Definition:
    """Of rows that are finite or -inf, in 64 bits: logp, p, entropy, and how far log(sum) may be off."""

    def __init__(self, x, scale):
        self.x = x.double()
        d = (self.x - self.x.amax(2, keepdim=True)) * scale
        d = torch.where(d.isnan(), -INF, d)                  # rows of nothing but -inf
        self.d = d.clamp(min=-1e4)
        e = torch.exp(d)
        s = e.sum(2, keepdim=True)
        self.empty = (s == 0.0)[..., 0]
        s = torch.where(s == 0.0, 1.0, s)
        self.log_sum = torch.log(s)
        self.p = e / s
        self.logp = d - self.log_sum
        far = (self.p * -self.d).sum(2, keepdim=True)        # mean distance to the largest
        far2 = (self.p * self.d ** 2).sum(2, keepdim=True)
        self.entropy = (self.log_sum + far)[..., 0] * ~self.empty
        vocab = x.shape[2]
        # exponentials: two steps each and three of their exponent, for every time that the largest so far changed; additions of a thread (of 64 for short rows),
        # lanes, waves, workgroups
        moves, adds = 16 + vocab / 8192, 96 + vocab / 256
        self.off_log_sum = U * (3 * far + 4 * moves + adds + 2 * self.log_sum.abs())
        self.off_entropy = (self.off_log_sum + far * U * (3 * far + 4 * moves + adds) + U * (3 * far2 + (4 * moves + adds + 4) * far))[..., 0]

    def off_logp(self):
        return U * (3 * self.d.abs() + 2 * self.logp.clamp(min=-1e4).abs()) + self.off_log_sum


def close(got, want, off, what):
    same = (got.double() == want) | (got.double().isnan() & want.isnan())
    far = torch.where(same, 0.0, (got.double() - want).abs() - off - HALF[got.dtype] * (want.abs() + off) - 1e-37)
    assert bool((far <= 0.0).all()), (what, float(far.nan_to_num(nan=INF).max()))


def ordered(x, top):
    """The first `top` tokens by logit, equal ones by number; -1 for logits of -inf."""
    order = torch.sort(x, dim=2, descending=True, stable=True).indices[..., :top]
    order = torch.nn.functional.pad(order, (0, top - order.shape[2]), value=-1)
    return torch.where(x.gather(2, order.clamp(min=0)) > -INF, order, -1)


def check_scores(values, dtype, targets, top=0, scale=1.0, lengths=None, gap=0, skip=0):
    n, tokens, vocab = values.shape
    x, _ = rows(values, dtype, gap, skip)
    desc = desc_of(x, top=top, scale=scale)
    f32 = lambda *shape: torch.full(shape, 7.0, device="cuda:0")
    lp, h, stats = f32(n, tokens), f32(n, tokens), f32(n, tokens, 2)
    tl, tt = (f32(n, tokens, top), torch.full((n, tokens, top), 7, dtype=torch.int32, device="cuda:0")) if top else (None, None)
    need = dp.dp_token_logprobs_workspace_bytes(desc)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda:0")
    dp.dp_token_logprobs(desc, x, targets, lp, h, stats, tl, tt, ws, lengths=lengths, ws_bytes=need)
    assert bool((ws[need:] == 0xA5).all())
    there, ref = there_of(lengths, n, tokens), Definition(x, scale)
    case = (tuple(values.shape), dtype, top, scale, gap, skip)
    t = targets.long()
    scored = there & (t >= 0) & (t < vocab)
    at = t.clamp(0, vocab - 1)[..., None]
    want = torch.where(scored, ref.logp.gather(2, at)[..., 0], 0.0)
    close(lp, want, ref.off_logp().gather(2, at)[..., 0], ("logprobs",) + case)
    close(h, torch.where(there, ref.entropy, 0.0), ref.off_entropy, ("entropy",) + case)
    assert bool((stats[~there] == 0.0).all())
    empty = there & ref.empty
    assert bool((stats[empty][:, 0] == 0.0).all()) and bool((stats[empty][:, 1] == INF).all())
    full = there & ~ref.empty
    assert torch.equal(stats[full][:, 0].double(), ref.x.amax(2)[full])
    close(stats[full][:, 1], ref.log_sum[..., 0][full], ref.off_log_sum[..., 0][full], ("stats",) + case)
    if top:
        order = torch.where(there[..., None], ordered(x, top), -1)
        assert torch.equal(tt.long(), order), ("top",) + case
        at = order.clamp(min=0)
        best = torch.where(order >= 0, ref.logp.gather(2, at), torch.where(there[..., None], -INF, 0.0))
        close(tl, best, ref.off_logp().gather(2, at), ("top logprobs",) + case)
    return lp, h, stats


def check_gradient(values, dtype, targets, scale=1.0, lengths=None, gap=0, skip=0, entropy=False, given=False, in_place=False, seed=0, out_skip=None):
    n, tokens, vocab = values.shape
    x, _ = rows(values, dtype, gap, skip)
    gen = torch.Generator("cuda:0").manual_seed(seed)
    a, b = torch.randn((n, tokens), generator=gen, device="cuda:0"), torch.randn((n, tokens), generator=gen, device="cuda:0") if entropy else None
    there, ref = there_of(lengths, n, tokens), Definition(x, scale)
    t = targets.long()
    scored = there & (t >= 0) & (t < vocab)
    live = there & ~ref.empty
    a64 = torch.where(scored & live, a.double(), 0.0)[..., None]
    b64 = torch.where(live, b.double(), 0.0)[..., None] if entropy else torch.zeros_like(a64)
    at = t.clamp(0, vocab - 1)[..., None]
    p, logp = torch.where(live[..., None], ref.p, 0.0), ref.logp.clamp(min=-1e4)
    own = torch.zeros_like(p).scatter_(2, at, torch.where(scored[..., None], 1.0, 0.0).double())
    rest = -torch.expm1(logp)
    want = scale * (a64 * torch.where(own > 0, rest, -p) - b64 * p * (logp + ref.entropy[..., None]))
    off_p = p * (ref.off_logp() + 4 * U + 2 * U * logp.abs())
    off = a64.abs() * (off_p + 4 * U * torch.where(own > 0, rest, p)) + b64.abs() * (off_p * (logp + ref.entropy[..., None]).abs()
          + p * (ref.off_logp() + ref.off_entropy[..., None] + 4 * U * (logp.abs() + ref.entropy[..., None])))
    off = scale * off + 4 * U * want.abs() + scale * (a64.abs() + b64.abs() * (ref.entropy[..., None] + 90)) * 2.0 ** -125      # (exponentials below 2^-126 are zeros)
    desc = desc_of(x, scale=scale)
    need = dp.dp_token_logprobs_workspace_bytes(desc)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda:0")
    stats = h = None
    if given:
        stats, h = torch.empty((n, tokens, 2), device="cuda:0"), torch.empty((n, tokens), device="cuda:0") if entropy else None
        dp.dp_token_logprobs(desc, x, None, None, h, stats, None, None, ws, lengths=lengths, ws_bytes=need)
    lp = torch.full((n, tokens), 7.0, device="cuda:0")
    out, around = (x, None) if in_place else rows(torch.full_like(values, 3.0), dtype, gap, skip if out_skip is None else out_skip)
    dp.dp_token_logprobs_backward(desc, x, targets, stats, a, out, ws, entropy=h, d_entropy=b, logprobs=lp, lengths=lengths, ws_bytes=need)
    case = (tuple(values.shape), dtype, scale, gap, skip, entropy, given, in_place)
    close(out, torch.where(there[..., None], want, 0.0), off, ("dlogits",) + case)
    close(lp, torch.where(scored, ref.logp.gather(2, at)[..., 0], 0.0), ref.off_logp().gather(2, at)[..., 0], ("logprobs",) + case)
    assert bool((out[~live] == 0.0).all()) and bool((ws[need:] == 0xA5).all())
    if around is not None:
        out.fill_(7.0)
        assert bool((around == 7.0).all())


def data(n, tokens, vocab, seed, size=3.0):
    gen = torch.Generator("cuda:0").manual_seed(seed)
    x = torch.randn((n, tokens, vocab), generator=gen, device="cuda:0") * size + torch.randn((n, tokens, 1), generator=gen, device="cuda:0") * 50
    t = torch.randint(0, vocab, (n, tokens), generator=gen, device="cuda:0", dtype=torch.int32)
    if tokens > 2:
        t[0, 1], t[-1, -1] = -1, vocab
    return x, t


# every kernel, just within and just beyond what a row's threads hold
VOCABS = [1, 2, 7, 8, 9, 31, 100, 511, 512, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16383, 16384, 16385, 32767, 32768, 32769, 50021,
          65535, 65536, 65537, 131071, 131072, 131073, 200003]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies(vocab, dtype):
    shapes = [(1, 1), (3, 5)] + ([(7, 75)] if vocab <= 70000 else [(2, 256)])      # few rows, and enough that each has a workgroup of its own
    for i, (n, tokens) in enumerate(shapes):
        x, t = data(n, tokens, vocab, vocab + i)
        scale = (1.0, 0.7, 1.25)[i]
        lengths = torch.tensor([5, 0, 2], dtype=torch.int32, device="cuda:0") if i == 1 else None
        check_scores(x, dtype, t, (0, 3, 0)[i], scale, lengths)
        check_gradient(x, dtype, t, scale, lengths, entropy=i == 0)
        if i == 1:
            check_gradient(x, dtype, t, scale, lengths, given=True)
            check_gradient(x, dtype, t, scale, lengths, given=True, entropy=True)
        if i == 2:
            check_gradient(x, dtype, t, scale, lengths, entropy=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,gap,skip", [(9, 0, 1), (100, 1, 0), (101, 0, 0), (1001, 2, 1), (2001, 1, 1), (9001, 0, 3), (9000, 3, 0), (40001, 0, 1), (66001, 1, 0)], ids=str)
def test_rows_that_begin_anywhere(vocab, gap, skip, dtype):
    for n, tokens in ((2, 3), (130, 4)) if vocab < 20000 else ((2, 3), (2, 260)):
        x, t = data(n, tokens, vocab, vocab)
        lengths = torch.full((n,), tokens, dtype=torch.int32, device="cuda:0")
        lengths[-1] = 1
        check_scores(x, dtype, t, 2, 1.0, lengths, gap, skip)
        for in_place in (False, True):
            check_gradient(x, dtype, t, 1.0, lengths, gap, skip, in_place=in_place)
            check_gradient(x, dtype, t, 1.0, lengths, gap, skip, in_place=in_place, given=True, entropy=True)
        check_gradient(x, dtype, t, 1.0, lengths, gap, skip, out_skip=skip + 1)      # results whose rows begin elsewhere in a dword
        check_gradient(x, dtype, t, 1.0, lengths, gap, skip, out_skip=skip + 1, given=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [1, 2, 31, 32])
@pytest.mark.parametrize("n,tokens,vocab", [(2, 3, 5), (2, 3, 33), (3, 200, 300), (2, 2, 9000), (1, 1, 131072), (5, 110, 9000), (1, 1, 200000)], ids=str)
def test_alternatives(n, tokens, vocab, top, dtype):
    """Ordinary rows, rows of a few values (ties to the lowest number), rows of one value, rows with logits of -inf, rows in order."""
    x, t = data(n, tokens, vocab, top)
    check_scores(x, dtype, t, top)
    check_scores(torch.round(x * 0.2), dtype, t, top)
    check_scores(torch.full_like(x, -3.5), dtype, t, top)
    some = torch.rand(x.shape, generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0") < 0.5
    check_scores(torch.where(some, x, -INF), dtype, t, top)
    few = torch.full_like(x, -INF)
    few[..., vocab // 2] = 2.0
    few[..., vocab - 1] = 2.0
    check_scores(few, dtype, t, top)
    line = torch.arange(vocab, device="cuda:0", dtype=torch.float32).expand_as(x) * 2.0 ** -6
    check_scores(line, dtype, t, top)
    check_scores(-line, dtype, t, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,tokens,vocab", [(3, 4, 50), (130, 4, 3000), (130, 4, 9000), (2, 3, 20000), (2, 260, 40000), (2, 260, 140000)], ids=str)
def test_masked_logits(n, tokens, vocab, dtype):
    """-inf and the type's lowest value for tokens that must not come; rows that are all masked; a single token that is left."""
    x, t = data(n, tokens, vocab, 3)
    gone = torch.rand(x.shape, generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0") < 0.9
    for low in (-INF, torch.finfo(dtype).min):
        y = torch.where(gone, low, x)
        y[:, 1] = low
        y[:, 2] = low
        y[:, 2, vocab - 1] = 1.0
        check_scores(y, dtype, t, 4)
        check_gradient(y, dtype, t, entropy=True)
        check_gradient(y, dtype, t, entropy=True, given=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,tokens,vocab", [(3, 6, 50), (100, 6, 3000), (100, 6, 9000), (3, 6, 20000), (3, 180, 40000), (3, 180, 140000)], ids=str)
def test_broken_rows_and_rows_beyond_the_lengths(n, tokens, vocab, dtype):
    x, t = data(n, tokens, vocab, 5)
    t[0, :3] = torch.tensor([0, 1, 2])
    x = x.to(dtype)
    lengths = torch.full((n,), tokens, dtype=torch.int32, device="cuda:0")
    lengths[1], lengths[2] = tokens - 1, 0
    there = there_of(lengths, n, tokens)
    desc, top = desc_of(x), desc_of(x, top=5)
    ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc), dp.dp_token_logprobs_workspace_bytes(top)), dtype=torch.uint8, device="cuda:0")
    weights = torch.randn((n, tokens), generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0")

    def all_of(x, weights):
        lp, h, stats = torch.empty((n, tokens), device="cuda:0"), torch.empty((n, tokens), device="cuda:0"), torch.empty((n, tokens, 2), device="cuda:0")
        tl, tt = torch.empty((n, tokens, 5), device="cuda:0"), torch.empty((n, tokens, 5), dtype=torch.int32, device="cuda:0")
        dp.dp_token_logprobs(top, x, t, lp, h, stats, tl, tt, ws, lengths=lengths)
        grads = [torch.empty_like(x) for _ in range(2)]
        dp.dp_token_logprobs_backward(desc, x, t, None, weights, grads[0], ws, d_entropy=weights, lengths=lengths)
        dp.dp_token_logprobs_backward(desc, x, t, stats, weights, grads[1], ws, entropy=h, d_entropy=weights, lengths=lengths)
        return [lp, h, stats, tl, tt] + grads
    clean = all_of(x, weights)
    bad = x.clone()
    bad[0, 0, 5], bad[0, 1, vocab - 1], bad[0, 2, 3] = math.nan, INF, math.nan
    bad[0, 2, 4] = -INF
    bad[~there] = math.nan
    other = torch.where(there, weights, math.nan)
    broken = all_of(bad, other)
    for i, (a, b) in enumerate(zip(clean, broken)):
        if i == 4:
            assert bool((b[0, :3] == -1).all())
        elif i == 3 or i >= 5:
            assert bool(b[0, :3].isnan().all()), i
        else:
            assert bool(b[0, :3].isnan().all()), i
        a[0, :3] = 0
        b[0, :3] = 0
        assert torch.equal(a, b), i


def test_rows_without_a_target_take_no_weight():
    x, _ = data(4, 5, 700, 6)
    t = torch.full((4, 5), -1, dtype=torch.int32, device="cuda:0")
    t[1] = 1 << 30
    desc = desc_of(x)
    ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc)), dtype=torch.uint8, device="cuda:0")
    weights, out, lp = torch.full((4, 5), math.nan, device="cuda:0"), torch.empty_like(x), torch.full((4, 5), 7.0, device="cuda:0")
    dp.dp_token_logprobs_backward(desc, x, t, None, weights, out, ws, logprobs=lp)
    assert bool((out == 0.0).all()) and bool((lp == 0.0).all())


def test_certain_targets_keep_their_small_gradients():
    """p of the target within 2^-20 of 1: its derivative, 1 - p, to fp32's digits and not to p's."""
    n, vocab = 8, 4000
    x = torch.zeros((1, n, vocab), device="cuda:0")
    x[0, :, 17] = 20.0 + torch.arange(n, device="cuda:0")
    t = torch.full((1, n), 17, dtype=torch.int32, device="cuda:0")
    desc = desc_of(x)
    ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc)), dtype=torch.uint8, device="cuda:0")
    out = torch.empty_like(x)
    dp.dp_token_logprobs_backward(desc, x, t, None, torch.ones((1, n), device="cuda:0"), out, ws)
    want = -torch.expm1(torch.log_softmax(x.double(), 2)[..., 17])
    # log(1 + small) of a sum that holds 1: half a step of 1, 2^-24, and the additions of a thread and of lanes beyond it, where small parts meet 1
    assert bool(((out[..., 17].double() - want).abs() <= 20 * U).all())


def test_gradient_against_differences():
    n, tokens, vocab, scale = 2, 3, 57, 0.8
    x, t = data(n, tokens, vocab, 9)
    gen = torch.Generator("cuda:0").manual_seed(2)
    a, b, step = (torch.randn(s, generator=gen, device="cuda:0") for s in ((n, tokens), (n, tokens), (n, tokens, vocab)))
    desc = desc_of(x, scale=scale)
    ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc)), dtype=torch.uint8, device="cuda:0")
    out = torch.empty_like(x)
    dp.dp_token_logprobs_backward(desc, x, t, None, a, out, ws, d_entropy=b)
    scored = (t >= 0) & (t < vocab)

    def value(x):
        logp = torch.log_softmax(x * scale, 2)
        own = logp.gather(2, t.long().clamp(0, vocab - 1)[..., None])[..., 0]
        return torch.where(scored, a.double() * own, 0.0) - b.double() * (logp.exp() * logp).sum(2)
    h = 1e-5
    slope = (value(x.double() + h * step) - value(x.double() - h * step)) / (2 * h)
    along = (out.double() * step).sum(2)
    # differences are off by h^2 times a third derivative, gradients by 2^-24 of logits of order 100 in 57 terms
    assert bool(((along - slope).abs() <= 1e-4 * (1.0 + slope.abs())).all())


@pytest.mark.parametrize("n,tokens,vocab", [(4, 1, 30000), (6, 100, 3000)], ids=str)
def test_recorded_and_on_another_stream(n, tokens, vocab):
    """Replays on new inputs, with eager calls between them, and two recorded calls that use one workspace in turn."""
    x, t = data(n, tokens, vocab, 4)
    x = x.to(torch.bfloat16)
    desc, top = desc_of(x), desc_of(x, top=6)
    ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc), dp.dp_token_logprobs_workspace_bytes(top)), dtype=torch.uint8, device="cuda:0")
    f32 = lambda *shape: torch.empty(shape, device="cuda:0")
    lp, h, stats, tl, lp2 = f32(n, tokens), f32(n, tokens), f32(n, tokens, 2), f32(n, tokens, 6), f32(n, tokens)
    tt, weights, grads = torch.empty((n, tokens, 6), dtype=torch.int32, device="cuda:0"), torch.ones((n, tokens), device="cuda:0"), [torch.empty_like(x) for _ in range(2)]
    outputs = [lp, h, stats, tl, tt, lp2] + grads

    def call(stream=None):
        dp.dp_token_logprobs(top, x, t, lp, h, stats, tl, tt, ws, stream=stream)
        dp.dp_token_logprobs_backward(desc, x, t, stats, weights, grads[0], ws, entropy=h, d_entropy=weights, stream=stream)
        dp.dp_token_logprobs_backward(desc, x, t, None, weights, grads[1], ws, logprobs=lp2, stream=stream)

    def results():
        torch.cuda.synchronize()
        return [o.clone() for o in outputs]
    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            call()
    side = torch.cuda.Stream()
    for seed in range(4):
        x.copy_(data(n, tokens, vocab, 100 + seed)[0])
        call()
        eager = results()
        for replay in [g.replay for g in graphs] + [lambda: call(side)]:
            for o in outputs:
                o.zero_()
            torch.cuda.synchronize()
            replay()
            assert all(torch.equal(a, b) for a, b in zip(eager, results()))


def test_offsets_beyond_2_to_the_32():
    """The last rows of a tensor of 4.6 billion logits against the same rows by themselves."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 30 * 2 ** 30:
        pytest.skip("30 GiB of device memory are not free")
    tokens, vocab, last = 70000, 65600, 300
    x = torch.zeros((1, tokens, vocab), dtype=torch.bfloat16, device="cuda:0")
    values, t = data(1, last, vocab, 1)
    x[:, -last:] = values
    targets = torch.zeros((1, tokens), dtype=torch.int32, device="cuda:0")
    targets[:, -last:] = t
    alone = x[:, -last:].clone()

    def run(x, t):
        tokens = x.shape[1]
        desc, top = desc_of(x), desc_of(x, top=3)
        ws = torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc), dp.dp_token_logprobs_workspace_bytes(top)), dtype=torch.uint8, device="cuda:0")
        lp, h = torch.empty((1, tokens), device="cuda:0"), torch.empty((1, tokens), device="cuda:0")
        tl, tt = torch.empty((1, tokens, 3), device="cuda:0"), torch.empty((1, tokens, 3), dtype=torch.int32, device="cuda:0")
        dp.dp_token_logprobs(top, x, t, lp, h, None, tl, tt, ws)
        grad = torch.empty_like(x)
        dp.dp_token_logprobs_backward(desc, x, t, None, torch.ones((1, tokens), device="cuda:0"), grad, ws)
        return lp[:, -last:].clone(), h[:, -last:].clone(), tl[:, -last:].clone(), tt[:, -last:].clone(), grad[:, -last:].clone()
    whole, part = run(x, targets), run(alone, t)
    assert torch.equal(whole[3], part[3])
    for a, b in zip(whole, part):                    # (rows shared by workgroups are added up in another order)
        assert bool(((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 2.0 ** -14).all())


def test_more_rows_than_a_launch_has_room_for():
    """33.5 million rows of two logits, and normalisations of 8.4 million examples of one token."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 20 * 2 ** 30:
        pytest.skip("20 GiB of device memory are not free")
    tokens = (1 << 25) + 4100
    gen = torch.Generator("cuda:0").manual_seed(1)
    x = torch.randn((1, tokens, 2), generator=gen, device="cuda:0")
    t = torch.randint(0, 2, (1, tokens), generator=gen, device="cuda:0", dtype=torch.int32)
    desc = desc_of(x)
    lp, lp2, stats, one, ws = torch.empty((1, tokens), device="cuda:0"), torch.empty((1, tokens), device="cuda:0"), torch.empty((1, tokens, 2), device="cuda:0"), torch.ones((1, tokens), device="cuda:0"), torch.empty(max(16, dp.dp_token_logprobs_workspace_bytes(desc)), dtype=torch.uint8, device="cuda:0")
    grads = [torch.empty_like(x) for _ in range(2)]
    dp.dp_token_logprobs(desc, x, t, lp, None, stats, None, None, ws)
    dp.dp_token_logprobs_backward(desc, x, t, None, one, grads[0], ws, logprobs=lp2)
    dp.dp_token_logprobs_backward(desc, x, t, stats, one, grads[1], ws)
    for part in (slice(0, 5000), slice(tokens // 2, tokens // 2 + 5000), slice(tokens - 5000, tokens)):
        logp = torch.log_softmax(x[:, part].double(), 2)
        own = logp.gather(2, t[:, part].long()[..., None])
        assert bool(((lp[:, part] - own[..., 0]).abs() <= 1e-5).all()) and bool(((lp2[:, part] - own[..., 0]).abs() <= 1e-5).all())
        want = torch.zeros_like(logp).scatter_(2, t[:, part].long()[..., None], 1.0) - logp.exp()
        for g in grads:
            assert bool(((g[:, part] - want).abs() <= 1e-5).all())
    n = (1 << 23) + 100
    x, dy = torch.randn((n, 1, 8), generator=gen, device="cuda:0"), torch.randn((n, 1, 8), generator=gen, device="cuda:0")
    desc = dp.NormDesc(in_dtype=dp.DP_F32, n=n, tokens=1, features=8, rms=0, eps=1e-5, row_stride=8)
    y, dx, g_w, g_b, sq = torch.empty_like(x), torch.empty_like(x), torch.empty((n, 8), device="cuda:0"), torch.empty((n, 8), device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(dp.dp_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dp.dp_layer_norm(desc, x, None, None, y)
    dp.dp_layer_norm_backward(desc, x, None, dy, dx, g_w, g_b, sq, ws)
    assert torch.equal(g_b, dy[:, 0])
    for part in (slice(0, 5000), slice(n - 5000, n)):
        d = x[part, 0].double() - x[part, 0].double().mean(1, keepdim=True)
        r = 1.0 / ((d ** 2).mean(1, keepdim=True) + 1e-5).sqrt()
        xhat, a = d * r, dy[part, 0].double()
        assert bool(((y[part, 0] - xhat).abs() <= 1e-4).all())
        assert bool(((g_w[part] - a * xhat).abs() <= 1e-4 * (1 + a.abs())).all())
        want = r * (a - a.mean(1, keepdim=True) - xhat * (a * xhat).mean(1, keepdim=True))
        assert bool(((dx[part, 0] - want).abs() <= 1e-4 * (1 + r * a.abs().amax(1, keepdim=True))).all())
        s = (g_w[part].double() ** 2 + g_b[part].double() ** 2).sum(1)
        assert bool(((sq[part] - s).abs() <= 1e-5 * s).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,top", [(3, 36864, 1), (5, 36864, 3), (7, 45060, 5), (2, 53251, 31)], ids=str)
def test_odd_numbers_of_workgroups_and_alternatives(n, vocab, top, dtype):
    """Rows that 9, 11 and 13 workgroups share, with odd numbers of alternatives."""
    gen = torch.Generator("cuda:0").manual_seed(vocab + top)
    values = torch.randn((n, 1, vocab), generator=gen, device="cuda:0") * 3.0
    targets = torch.randint(0, vocab, (n, 1), generator=gen, device="cuda:0", dtype=torch.int32)
    check_scores(values, dtype, targets, top=top)
    check_scores(values, dtype, targets, top=top, lengths=torch.tensor([1, 0, 1, 1, 0, 1, 1][:n], dtype=torch.int32, device="cuda:0"))
