"""The read-out block's private sums against plain per-example gradients in 64 bits, from the block's own intermediate values; its gradients against automatic
differentiation of the whole block; its step; its form for single tokens; a model of an attention block and it."""
import math

import numpy as np
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8                      # half a step of fp32, of bf16
N, TOKENS, WIDTH, VOCAB = 5, 37, 90, 333


def block_of(**more):
    fields = dict(clip_c=0.7, sigma=0.0, total_batch=2 * N, lr=0.5, momentum=0.9, seed=3, device="cuda:0")
    block = dp.PrivateReadout(N, TOKENS, WIDTH, VOCAB, **{**fields, **more})
    gen = torch.Generator().manual_seed(1)
    block.weights[0].copy_(1.0 + 0.3 * torch.randn(WIDTH, generator=gen))
    if not block.rms:
        block.weights[1].copy_(0.2 * torch.randn(WIDTH, generator=gen))
    return block


def data(seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((N, TOKENS, WIDTH), generator=gen).to(torch.bfloat16)
    targets = torch.randint(0, VOCAB, (N, TOKENS), generator=gen, dtype=torch.int32)
    targets[0, 3], targets[2, 0] = -1, VOCAB
    lengths = torch.tensor([TOKENS, 20, 1, 0, 33], dtype=torch.int32)
    weights = -torch.rand((N, TOKENS), generator=gen)
    weights[1] *= 1e-4                                # an example that is not clipped
    late = torch.arange(TOKENS)[None] >= lengths[:, None]
    x[late], weights[late] = math.nan, math.nan      # what is beyond the lengths does not matter
    return x.cuda(), targets.cuda(), lengths.cuda(), weights.cuda()


def double(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("rms", [False, True])
def test_private_sums_and_step(rms):
    block = block_of(rms=rms)
    x, targets, lengths, weights = data()
    _, dx = block.train(x, targets, weights, lengths)
    there = np.arange(TOKENS)[None] < lengths.cpu().numpy()[:, None]
    assert float(dx[~torch.from_numpy(there).cuda()].abs().max()) == 0.0
    back = torch.empty((N * TOKENS, WIDTH), dtype=torch.float32, device="cuda:0")
    dp.dp_checkpoint_read(*block.kept, back)
    values, d = double(back).reshape(N, TOKENS, WIDTH), double(block.dlogits)
    assert (d[~there] == 0.0).all() and (values[~there] == 0.0).all()
    projection = np.matmul(d.transpose(0, 2, 1), values)
    room = (TOKENS + 8) * U * np.matmul(np.abs(d).transpose(0, 2, 1), np.abs(values))
    affine = double(block.g_affine)
    squares, affine_squares = (projection ** 2).sum((1, 2)), (affine ** 2).sum(1)
    # the projection's norm may go by way of Gram matrices, whose sums of products are off by their terms
    gram = np.matmul(np.abs(d), np.abs(d).transpose(0, 2, 1)) * np.matmul(np.abs(values), np.abs(values).transpose(0, 2, 1))
    slack = (2 * np.abs(projection) * room + room ** 2).sum((1, 2)) + (2 * VOCAB + TOKENS ** 2) * U * gram.sum((1, 2)) + 500 * U * (squares + affine_squares)
    norms = squares + affine_squares
    assert (np.abs(double(block.total_sqnorm) - norms) <= slack + 1e-30).all()
    f = np.array([1.0 if v == 0.0 else min(1.0, block.clip_c / math.sqrt(v)) for v in norms])
    assert (f < 1.0).sum() >= 2 and (f == 1.0).sum() >= 2
    rel = np.where(norms > 0.0, slack / np.maximum(norms, 1e-30), 0.0) + 8 * U
    want = (f[:, None, None] * projection).sum(0)
    allowed = (f[:, None, None] * (3 * room + rel[:, None, None] * np.abs(projection) + (N + 4) * 2 * U * np.abs(projection))).sum(0)
    assert (np.abs(double(block.sums[-1]) - want) <= allowed + 1e-30).all()
    stride = affine.shape[1]
    got, want = double(block.acc[:stride]), (f[:, None] * affine).sum(0)
    assert (np.abs(got - want) <= ((rel + 16 * U)[:, None] * np.abs(f[:, None] * affine)).sum(0) + 1e-30).all()
    share = f[0] ** 2 * norms[0]
    assert share <= block.clip_c ** 2 * (1 + 1e-12)
    before, acc = double(block.theta), double(block.acc)
    block.step(0)
    step, after = 0.5 * acc / (2 * N), double(block.theta)
    assert (np.abs(after - (before - step)) <= 4 * U * np.abs(step) + U * np.abs(after)).all()
    assert float(block.acc.abs().max()) == 0.0 and float(block.velocity.abs().max()) > 0.0


@pytest.mark.parametrize("rms", [False, True])
def test_gradients_are_those_of_the_block(rms):
    block = block_of(rms=rms, clip_c=math.inf, scale=0.8)
    x, targets, lengths, weights = data(5)
    weights[1] *= 1e4
    there = torch.arange(TOKENS)[None] < lengths.cpu()[:, None]
    y, dx = block.train(x, targets, weights, lengths)
    params = [w.detach().cpu().to(torch.bfloat16 if i == len(block.weights) - 1 else torch.float32).double().requires_grad_() for i, w in enumerate(block.weights)]
    xs = torch.where(there[..., None], x.cpu().double(), 0.0).requires_grad_()
    dev = xs if rms else xs - xs.mean(2, keepdim=True)
    normed = dev / ((dev ** 2).mean(2, keepdim=True) + 1e-5).sqrt() * params[0] + (0.0 if rms else params[1])
    logp = torch.log_softmax(normed @ params[-1].t() * 0.8, 2)
    t = targets.cpu().long()
    scored = there & (t >= 0) & (t < VOCAB)
    own = torch.where(scored, logp.gather(2, t.clamp(0, VOCAB - 1)[..., None])[..., 0], 0.0)
    torch.where(scored, own * weights.cpu().double(), 0.0).sum().backward()
    # the projection's gradient meets values of 8 bits (a rounding is at most 2^-4 of a value); the others go through bf16 alone, three roundings deep
    for name, got, ref, most in [("y", y, own, 2.0 ** -6), ("dx", dx, xs.grad, 2.0 ** -5)] + [
            (str(i), s, w.grad, 0.0625 if i == len(params) - 1 else 2.0 ** -5) for i, (s, w) in enumerate(zip(block.sums, params))]:
        got, ref = double(got), ref.detach().numpy()
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert off <= most, (name, off)


def test_autograd_the_passes_one_by_one_and_both_at_once_agree():
    x, targets, lengths, weights = data(2)
    blocks = [block_of() for _ in range(3)]
    leaf = x.clone().requires_grad_()
    y = blocks[0].logprobs(leaf, targets, lengths)
    scored = y.detach() != 0.0
    torch.where(scored, y * weights, 0.0).sum().backward()
    plain = blocks[1].logprobs(x, targets, lengths)
    assert not plain.requires_grad and torch.equal(plain, y)
    dx = blocks[1].backward(torch.where(scored, weights, 0.0))
    assert torch.equal(dx, leaf.grad) and torch.equal(blocks[0].acc, blocks[1].acc) and float(dx.abs().max()) > 0.0
    both, dx2 = blocks[2].train(x, targets, weights, lengths)
    # the same sums, added up in another order
    assert bool(((both - plain).abs() <= 64 * U * (1.0 + plain.abs())).all())
    for a, b in ((dx2, dx), (blocks[2].acc, blocks[1].acc)):
        assert float((a - b).norm()) <= 2.0 ** -7 * float(b.norm())


def test_a_pass_that_the_block_no_longer_holds_is_refused():
    x, targets, lengths, weights = data(2)
    block = block_of()
    with pytest.raises(RuntimeError, match="holds no forward pass"):
        block.backward(weights)
    clean = torch.nan_to_num(x)
    first = block.logprobs(clean.clone().requires_grad_(), targets, lengths)
    second = block.logprobs(clean.clone().requires_grad_(), targets, lengths)
    with pytest.raises(RuntimeError, match="no longer holds"):
        first.backward(weights)
    second.backward(weights, retain_graph=True)
    acc = block.acc.clone()
    with pytest.raises(RuntimeError, match="no longer holds"):
        second.backward(weights)
    with pytest.raises(RuntimeError, match="holds no forward pass"):
        block.backward(weights)
    assert torch.equal(block.acc, acc)
    for bad in (dict(x=x.float()), dict(targets=targets.long()), dict(targets=targets.cpu()), dict(lengths=lengths.long()), dict(x=x[:, :-1])):
        with pytest.raises(ValueError):
            block.logprobs(**{**dict(x=x, targets=targets, lengths=lengths), **bad})


def test_next_tokens_are_those_of_the_last_places():
    block = block_of(scale=0.5)
    x, targets, _, _ = data(9)
    x = torch.nan_to_num(x)
    last = x[:, -1].contiguous()
    tokens, best = block.next_tokens(last, 7)
    targets[:, -1] = tokens[:, 2]
    y = block.logprobs(x, targets)
    # (the library's products over another number of rows may round otherwise)
    assert bool(((best[:, 2] - y[:, -1]).abs() <= 4 * HALF * (1.0 + y[:, -1].abs())).all())
    logits = block.logits[:, -1].float()
    kept = logits.gather(1, tokens.long())
    assert bool((kept[:, :-1] >= kept[:, 1:] - 2 * HALF * kept[:, 1:].abs()).all())
    assert bool((kept[:, -1:] + 2 * HALF * kept[:, -1:].abs() + 1e-3 >= logits.topk(7).values[:, -1:]).all())
    assert bool((best[:, :-1] >= best[:, 1:]).all())


def test_a_model_of_an_attention_block_and_the_readout():
    """Both trained in one pass of automatic differentiation: each block's accumulator is what its own backward pass makes of its part of the chain."""
    n, tokens, width, vocab = 4, 21, 64, 100
    gen = torch.Generator().manual_seed(4)
    x = torch.randn((n, tokens, width), generator=gen).to(torch.bfloat16).cuda()
    targets = torch.randint(0, vocab, (n, tokens), generator=gen, dtype=torch.int32).cuda()
    lengths = torch.tensor([tokens, 7, 0, 1], dtype=torch.int32, device="cuda:0")

    def model():
        return (dp.PrivateAttention(n, tokens, width, 4, clip_c=0.5, sigma=0.5, total_batch=n, lr=0.1, seed=2, buckets=8, max_distance=16, device="cuda:0"),
                dp.PrivateReadout(n, tokens, width, vocab, clip_c=0.5, sigma=0.5, total_batch=n, lr=0.1, seed=3, device="cuda:0"))
    attention, readout = model()
    leaf = x.clone().requires_grad_()
    y = readout.logprobs(attention.forward(leaf, lengths), targets, lengths)
    (-y.sum(1) / lengths.clamp(min=1)).sum().backward()
    one, two = model()
    z = two.logprobs(one.forward(x, lengths), targets, lengths)
    assert torch.equal(z, y)
    there = torch.arange(tokens, device="cuda:0")[None] < lengths[:, None]
    dx = one.backward(two.backward((-1.0 / lengths.clamp(min=1).float())[:, None].expand(n, tokens)))
    assert torch.equal(leaf.grad, dx) and torch.equal(attention.acc, one.acc) and torch.equal(readout.acc, two.acc)
    assert float(attention.acc.abs().max()) > 0.0 and float(readout.acc.abs().max()) > 0.0
    for block in (attention, readout):
        before = block.theta.clone()
        block.step(0)
        assert bool(block.theta.isfinite().all()) and not torch.equal(block.theta, before)
    assert bool((z[~there] == 0.0).all())


def test_a_recorded_pass():
    """Replays on new tokens, with eager passes of another block between them."""
    x, targets, lengths, weights = data(3)
    x, weights = torch.nan_to_num(x), torch.nan_to_num(weights)
    recorded, eager = block_of(), block_of()
    recorded.train(x, targets, weights, lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = recorded.train(x, targets, weights, lengths)
    for seed in range(4):
        new = data(20 + seed)
        for old, fresh in zip((x, targets, lengths, weights), new):
            old.copy_(torch.nan_to_num(fresh))
        recorded.acc.zero_()
        eager.acc.zero_()
        graph.replay()
        want = eager.train(x, targets, weights, lengths)
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(recorded.acc, eager.acc) and float(eager.acc.abs().max()) > 0.0
