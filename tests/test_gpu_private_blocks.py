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
