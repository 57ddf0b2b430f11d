"""The attention block's private sums against plain per-example gradients in 64 bits, from the block's own intermediate values; its gradients
against automatic differentiation of the whole block; its step; its form for single tokens."""
import math

import numpy as np
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -8                      # half a step of fp32, of bf16


def block_of(n=5, tokens=37, width=96, heads=3, **more):
    block = dp.PrivateAttention(n, tokens, width, heads, clip_c=1.5, sigma=0.0, total_batch=2 * n, lr=0.5, momentum=0.9, seed=3, buckets=16,
                                max_distance=20, device="cuda:0", **more)
    block.weights[4].copy_(torch.randn(16, heads, generator=torch.Generator().manual_seed(1)) * 0.5)
    return block


def data(block, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x, dy = (torch.randn((block.n, block.tokens, block.width), generator=gen).to(torch.bfloat16) for _ in range(2))
    dy[1] *= 1e-3                                     # an example that is not clipped
    lengths = torch.tensor([block.tokens, 20, 1, 0, 33], dtype=torch.int32)
    dy[torch.arange(block.tokens)[None] >= lengths[:, None]] = 0.0
    return x.cuda(), dy.cuda(), lengths.cuda()


def double(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("more", [{}, dict(causal=True, bidirectional=False)], ids=str)
def test_private_sums_and_step(more):
    block = block_of(**more)
    x, dy, lengths = data(block)
    n, T, H, W = block.n, block.tokens, block.heads, block.width
    block.forward(x, lengths)
    block.backward(dy)
    values = []
    for codes, scales in (block.inputs, block.mixed):
        back = torch.empty((n * T, W), dtype=torch.float32, device="cuda:0")
        dp.dp_checkpoint_read(codes, scales, back)
        values.append(double(back).reshape(n, T, W))
    ls = lengths.cpu().numpy()
    there = np.arange(T)[None] < ls[:, None]
    for v in values:
        v[~there] = 0.0
    per, room = [], []                                # per-example gradients, and what their own rounding can be
    for i, g in enumerate(block.grads):
        g = double(g) * there[..., None]
        xv = values[0 if i < 3 else 1]
        per.append(np.matmul(g.transpose(0, 2, 1), xv))
        room.append((T + 8) * U * np.matmul(np.abs(g).transpose(0, 2, 1), np.abs(xv)))
    p, d = double(block.probs), double(block.dprobs)
    bucket = np.array([[dp.dp_bias_bucket(block.bias, q - k) for k in range(T)] for q in range(T)])
    counts = there[:, None, :, None] & there[:, None, None, :] & (np.tril(np.ones((T, T), bool)) if more else np.ones((T, T), bool))
    p, d = np.where(counts, p, 0.0), np.where(counts, d, 0.0)
    dot = (p * d).sum(3, keepdims=True)
    dz = p * (d - dot)
    off = p * ((T + 2) * U * np.abs(p * d).sum(3, keepdims=True) + 3 * U * np.abs(d - dot)) + (2 * T + 64) * U * np.abs(dz)
    table, table_room = np.zeros((n, 16, H)), np.zeros((n, 16, H))
    for i in range(n):
        for h in range(H):
            table[i, :, h] = np.bincount(bucket.ravel(), dz[i, h].ravel(), 16)
            table_room[i, :, h] = np.bincount(bucket.ravel(), off[i, h].ravel(), 16)
    per.append(table)
    room.append(table_room)
    norms = sum((g.reshape(n, -1) ** 2).sum(1) for g in per)
    # a norm's error: its gradients' own, and fp32 sums of their squares; the Gram form of a projection's is off by the products' sums instead
    gram = np.zeros(n)
    for i, g in enumerate(block.grads):
        g = np.abs(double(g)) * there[..., None]
        xv = np.abs(values[0 if i < 3 else 1])
        gram += (np.matmul(g, g.transpose(0, 2, 1)) * np.matmul(xv, xv.transpose(0, 2, 1))).sum((1, 2))
    slack = sum((2 * np.abs(g) * r + r * r).reshape(n, -1).sum(1) for g, r in zip(per, room)) + (2 * W + T * T + 64) * U * gram + 5 * W * W * U * norms
    got = double(block.total_sqnorm)
    print("norms", got, "off", np.abs(got - norms), "room", slack)
    assert (np.abs(got - norms) <= slack + 1e-30).all()
    f = np.array([1.0 if v == 0.0 else min(1.0, block.clip_c / math.sqrt(v)) for v in norms])
    assert (f < 1.0).sum() >= 2 and (f == 1.0).sum() >= 2
    rel = np.where(norms > 0.0, slack / np.maximum(norms, 1e-30), 0.0) + 8 * U            # of a factor
    for g, r, acc in zip(per, room, block.sums):
        shape = (n,) + (1,) * (g.ndim - 1)
        want = (f.reshape(shape) * g).sum(0)
        # the factor is applied to sums or to values split into three bf16 parts: 2^-23 of each product more
        allowed = (f.reshape(shape) * (r * (1 + 4 * HALF) + rel.reshape(shape) * np.abs(g) + (n + 4) * 2 * U * np.abs(g) + 2 * r)).sum(0)
        wrong = np.abs(double(acc) - want) - allowed
        assert wrong.max() <= 1e-30, (wrong.max(), allowed.ravel()[wrong.argmax()])
    # clipped: the norm of one example's share is at most the bound
    share = sum(float((np.abs(f[0] * g[0]) ** 2).sum()) for g in per)
    assert share <= block.clip_c ** 2 * (1 + 1e-12)
    before, acc = double(block.theta), double(block.acc)
    block.step(0)
    after = double(block.theta)
    step = 0.5 * acc / (2 * n)
    assert (np.abs(after - (before - step)) <= 4 * U * np.abs(step) + U * np.abs(after)).all()
    assert float(block.acc.abs().max()) == 0.0
    assert float(block.velocity.abs().max()) > 0.0


def test_gradients_are_those_of_the_block():
    block = block_of()
    block.clip_c = math.inf                           # the plain sum of gradients
    x, dy, lengths = data(block, 5)
    y = block.forward(x, lengths)
    dx = block.backward(dy)
    n, T, H, W = block.n, block.tokens, block.heads, block.width
    weights = [w.detach().double().cpu().to(torch.bfloat16 if i < 4 else torch.float32).double().requires_grad_() for i, w in enumerate(block.weights)]
    xs = x.cpu().double().requires_grad_()
    heads = lambda v: v.view(n, T, H, W // H).transpose(1, 2)
    q, k, v = (heads(xs @ w.t()) for w in weights[:3])
    bucket = torch.tensor([[dp.dp_bias_bucket(block.bias, a - b) for b in range(T)] for a in range(T)])
    scores = q @ k.transpose(2, 3) * (W // H) ** -0.5 + weights[4][bucket].permute(2, 0, 1)
    there = torch.arange(T)[None] < lengths.cpu()[:, None]
    probs = torch.softmax(scores.masked_fill(~there[:, None, None, :], -1e300), 3) * (there[:, None, :, None] & there[:, None, None, :])
    want = (probs @ v).transpose(1, 2).reshape(n, T, W) @ weights[3].t()
    want.backward(dy.cpu().double())
    # values of 8 bits (a rounding is at most 2^-4 of a value) and of bf16, several products deep: an eighth, as a norm
    for name, got, ref in [("y", y, want), ("dx", dx, xs.grad)] + [("qkvo"[i] if i < 4 else "table", s, w.grad) for i, (s, w) in enumerate(zip(block.sums, weights))]:
        got, ref = double(got), ref.detach().numpy()
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        print(name, off)
        assert off <= 0.125, (name, off)


def test_last_token_is_the_block_s_last():
    block = block_of(causal=True, bidirectional=False)
    x, _, _ = data(block, 9)
    lengths = torch.tensor([block.tokens, 20, 1, 2, 33], dtype=torch.int32, device="cuda:0")
    y = block.forward(x, lengths)
    at = (lengths.long() - 1).clamp(min=0)
    rows = torch.arange(block.n, device="cuda:0")
    q = block.q.transpose(1, 2).reshape(block.n, block.tokens, block.width)[rows, at].contiguous()
    got, want = double(block.attend_last(q, block.k, block.v, lengths)), double(y[rows, at])
    # both round the scores, the probabilities and their products with v to bf16, once each, of sums that differ by their order
    assert np.linalg.norm(got - want) <= 4 * HALF * np.linalg.norm(want)
