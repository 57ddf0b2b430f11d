"""Private blocks of one model: their steps' noise."""
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu


def test_blocks_as_they_come_draw_different_noise():
    """Steps after no example at all leave the noise alone: no two tensors' are related, whichever blocks they belong to."""
    n, tokens, width, vocab = 2, 3, 64, 100
    fields = dict(clip_c=1.0, sigma=1.0, total_batch=1, lr=1.0, device="cuda:0")
    first = dp.PrivateAttention(n, tokens, width, 4, **fields)
    blocks = [first, dp.PrivateAttention(n, tokens, width, 4, first_tensor=first.next_tensor, **fields), dp.PrivateReadout(n, tokens, width, vocab, **fields)]
    noise = []
    for block in blocks:
        block.theta.zero_()
        block.step(3)
        noise += [-w.flatten().double() for w in block.weights]
    for i, a in enumerate(noise):
        for b in noise[:i]:
            k = min(a.numel(), b.numel())
            # the mean of k products of independent normals: 0 +- k^-1/2
            assert float((a[:k] * b[:k]).mean().abs()) <= 6.0 * k ** -0.5


@pytest.mark.parametrize("graph", [False, True], ids=["by hand", "autograd"])
@pytest.mark.parametrize("which", ["attention", "readout"])
def test_a_pass_back_is_over_the_targets_and_lengths_of_its_forward_pass(which, graph):
    """A loop that fills the same targets and lengths again before the pass back."""
    n, tokens, width, vocab = 4, 19, 64, 100
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((n, tokens, width), generator=gen).to(torch.bfloat16).cuda()
    d = torch.randn((n, tokens), generator=gen).cuda() if which == "readout" else torch.randn((n, tokens, width), generator=gen).to(torch.bfloat16).cuda()
    first, second = ((torch.randint(0, vocab, (n, tokens), generator=gen, dtype=torch.int32).cuda(), torch.tensor(v, dtype=torch.int32).cuda())
                     for v in ([tokens, 7, 0, 1], [3, tokens, 5, tokens]))

    def passes(refill):
        fields = dict(clip_c=0.5, sigma=0.0, total_batch=n, device="cuda:0")
        targets, lengths, leaf = first[0].clone(), first[1].clone(), x.clone().requires_grad_(graph)
        if which == "readout":
            block = dp.PrivateReadout(n, tokens, width, vocab, **fields)
            y = block.logprobs(leaf, targets, lengths)
        else:
            block = dp.PrivateAttention(n, tokens, width, 4, **fields)
            y = block.forward(leaf, lengths)
        if refill:
            targets.copy_(second[0])
            lengths.copy_(second[1])
        if graph:
            y.backward(d)
            return leaf.grad, block.acc
        return block.backward(d), block.acc
    kept, filled = passes(False), passes(True)
    assert float(kept[0].abs().max()) > 0.0 and float(kept[1].abs().max()) > 0.0
    assert torch.equal(kept[0], filled[0]) and torch.equal(kept[1], filled[1])


def test_an_input_that_was_written_to_is_refused():
    """The read-out holds its input as it is, without a copy: autograd's pass back says so."""
    n, tokens, width, vocab = 2, 5, 64, 100
    block = dp.PrivateReadout(n, tokens, width, vocab, clip_c=0.5, sigma=0.0, total_batch=n, device="cuda:0")
    leaf = torch.randn((n, tokens, width), device="cuda:0").to(torch.bfloat16).requires_grad_()
    x = leaf * 1.0
    y = block.logprobs(x, torch.zeros((n, tokens), dtype=torch.int32, device="cuda:0"))
    with torch.no_grad():
        x.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    assert float(block.acc.abs().max()) == 0.0
