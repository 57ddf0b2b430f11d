"""The attention block as a part of a model that automatic differentiation trains."""
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu

N, TOKENS, WIDTH, HEADS = 4, 21, 64, 4


def block_of():
    block = dp.PrivateAttention(N, TOKENS, WIDTH, HEADS, clip_c=0.5, sigma=0.0, total_batch=N, seed=2, buckets=8, max_distance=16, device="cuda:0")
    block.weights[4].copy_(torch.randn(8, HEADS, generator=torch.Generator().manual_seed(1)))
    return block


def data():
    gen = torch.Generator().manual_seed(4)
    x, dy = (torch.randn((N, TOKENS, WIDTH), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    return x, dy, torch.tensor([TOKENS, 7, 0, 1], dtype=torch.int32, device="cuda:0")


def test_gradient_of_the_input_is_that_of_the_whole_block():
    x, dy, lengths = data()
    plain, recorded = block_of(), block_of()
    y = plain.forward(x, lengths)
    assert not y.requires_grad
    dx = plain.backward(dy)
    assert not dx.requires_grad
    leaf = x.clone().requires_grad_()
    again = recorded.forward(leaf, lengths)
    assert torch.equal(again, y)
    (again * dy).sum().backward()
    assert torch.equal(leaf.grad, dx) and torch.equal(recorded.acc, plain.acc) and float(plain.acc.abs().max()) > 0.0


def test_layers_before_and_after_it_get_their_gradients():
    """A trained scale in front of the block and one behind it, against the block's own backward pass."""
    x, _, lengths = data()
    block = block_of()
    scale = torch.ones(WIDTH, dtype=torch.bfloat16, device="cuda:0", requires_grad=True)
    out = torch.full((WIDTH,), 0.5, dtype=torch.bfloat16, device="cuda:0", requires_grad=True)
    y = block.forward(x * scale, lengths)
    (y * out).sum().backward()
    plain = block_of()
    y0 = plain.forward(x, lengths)
    dx = plain.backward(torch.full_like(y0, 0.5))
    assert torch.equal(block.acc, plain.acc)
    # sums of bf16 products, rounded to bf16 once more: 2^-8 of the terms each
    for got, terms in ((scale.grad, x.double() * dx.double()), (out.grad, y0.double())):
        off = 2.0 ** -7 * terms.abs().sum((0, 1)) + 1e-6
        assert bool(((got.double() - terms.sum((0, 1))).abs() <= off).all())


def test_a_pass_that_the_block_no_longer_holds_is_refused():
    x, dy, lengths = data()
    block = block_of()
    first = block.forward(x.clone().requires_grad_(), lengths)
    second = block.forward(x.clone().requires_grad_(), lengths)
    with pytest.raises(RuntimeError, match="no longer holds"):
        first.backward(dy)
    assert float(block.acc.abs().max()) == 0.0
    second.backward(dy, retain_graph=True)
    acc = block.acc.clone()
    with pytest.raises(RuntimeError, match="no longer holds"):
        second.backward(dy)                          # the same examples would count twice
    assert torch.equal(block.acc, acc)


def test_serving_and_plain_passes_carry_no_graph():
    x, dy, lengths = data()
    block = block_of()
    leaf = x.clone().requires_grad_()
    with torch.no_grad():
        y = block.forward(leaf, lengths)
    assert not y.requires_grad
    assert not block.backward(dy.clone().requires_grad_()).requires_grad
    q = x[:, 0].contiguous().requires_grad_()
    k, v = (t.clone().requires_grad_() for t in (block.k, block.v))
    assert not block.attend_last(q, k, v, lengths).requires_grad
