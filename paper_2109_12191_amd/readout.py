"""What a token model ends in, trained privately: the last normalisation, the projection onto the vocabulary and the loss, on the token operators.

Per micro-step of `n` examples of up to `tokens` tokens:
    forward    dp_layer_norm of the input, dp_checkpoint_write of what it makes of it, the projection, dp_token_logprobs of the targets.  Kept for the backward
               pass: the input, one 8-bit checkpoint, the logits and two numbers a token
    backward   dp_token_logprobs_backward (into the logits' place), dp_checkpoint_example_grad of the projection (squared norms alone),
               dp_layer_norm_backward (the input's gradient, and each example's gradients of scale and shift with their squared norm), dp_norms, then
               dp_checkpoint_clip_accumulate and dp_clip_accumulate into the flat accumulator
and per optimiser step dp_add_noise_finalize_flat with the SGD update.  The projection's own products are the framework's user's, here torch's.

An example's gradient is that of its checkpoint's values, for the norm and for the clipped sum alike (PrivateAttention).  Clipping is by example, so the
derivatives that a backward pass starts from are those of a sum over examples, not of a mean.

logprobs' result carries a graph where its input requires a gradient: autograd's pass over it is `backward`, with the clipped sums of the parameters that
belong to it, and gives the input's gradient.  Elsewhere `backward` is called, or `train` for both passes at once, which is also what to record into a graph.  The
block holds the values of one forward pass, its targets and lengths among them, for one such pass back, and the input itself, which has to stay as it is until
then (autograd's pass refuses one that was written to).
"""
from __future__ import annotations

import torch

from . import binding as B


FIRST_TENSOR = 1 << 16               # a model's last block: behind the tensors of the blocks before it, which count theirs from zero


class _Recorded(torch.autograd.Function):
    """A forward pass that autograd knows of as a whole."""

    @staticmethod
    def forward(ctx, x, block, targets, lengths):
        y = block._logprobs(x, targets, lengths)
        ctx.block, ctx.passes = block, block.passes
        ctx.save_for_backward(x)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logprobs):
        if ctx.block.passes != ctx.passes:
            raise RuntimeError("the block no longer holds this forward pass: there was another one, or a pass back over it")
        ctx.saved_tensors                                  # (raises where x was written to)
        return ctx.block.backward(d_logprobs), None, None, None


class PrivateReadout:
    """Scale [width] and shift [width] of the normalisation (rms: no shift, no mean) and the projection [vocab, width], fp32 in one vector `theta`;
    activations and logits are bf16, log probabilities fp32.  Tokens beyond an example's length (int32 `lengths`, None: all there) count for nothing,
    whatever they hold; tokens whose target is none of 0 .. vocab - 1 are not scored.

    The noise of a tensor is a function of seed, step and its number, from first_tensor on: blocks of one model and one seed need numbers of their own, or two tensors get
    the same noise, which a difference takes out again.  A read-out's own begin far behind those of the blocks before it; a model of several gives each its first_tensor.

    clip_c bounds what an example adds to this block.  A model of several blocks releases all their updates, so an example's part in what is released is bounded by the square
    root of the sum of the blocks' clip_c squared (dp_group_clip_bounds shares a bound out): that is every block's clip_total, which its noise has sigma times of.  None:
    the block is the whole model."""

    def __init__(self, n: int, tokens: int, width: int, vocab: int, clip_c: float, sigma: float, total_batch: int, lr: float = 0.0, momentum: float = 0.0,
                 seed: int = 0, rms: bool = False, eps: float = 1e-5, scale: float = 1.0, device: str = "cuda",
                 first_tensor: int = FIRST_TENSOR, clip_total: float | None = None):
        if not 0 <= first_tensor < (1 << 32) - 3:
            raise ValueError(f"first_tensor {first_tensor} and those behind it are not numbers of 32 bits")
        self.n, self.tokens, self.width, self.vocab, self.rms = n, tokens, width, vocab, rms
        if clip_total is not None and not clip_total >= clip_c * (1.0 - 2.0 ** -23):          # (bounds are fp32 to the library)
            raise ValueError(f"clip_total {clip_total} does not cover this block's own clip_c {clip_c}")
        self.clip_total = clip_total
        self.clip_c, self.sigma, self.total_batch, self.lr, self.momentum, self.seed = clip_c, sigma, total_batch, lr, momentum, seed
        self.device = device
        affine = (width + 3) // 4 * 4
        shapes = [(width,), (width,), (vocab, width)] if not rms else [(width,), (vocab, width)]
        begins = [0, affine, 2 * affine] if not rms else [0, affine]
        total = begins[-1] + (vocab * width + 3) // 4 * 4
        f32 = dict(dtype=torch.float32, device=device)
        self.theta, self.acc, self.velocity = torch.zeros(total, **f32), torch.zeros(total, **f32), torch.zeros(total, **f32)
        sizes = [s[0] if len(s) == 1 else s[0] * s[1] for s in shapes]
        self.tensors = B.TensorTable(begins, sizes, range(first_tensor, first_tensor + len(begins)))
        self.next_tensor = first_tensor + len(begins)     # the first number that is none of this block's
        view = lambda flat: [flat[b:b + size].view(*shape) for b, size, shape in zip(begins, sizes, shapes)]  # noqa: E731
        self.weights, self.sums = view(self.theta), view(self.acc)
        self.weights[0].fill_(1.0)
        self.weights[-1].normal_(0.0, width ** -0.5, generator=torch.Generator(device=device).manual_seed(seed))
        self.norm = B.NormDesc(in_dtype=B.DP_BF16, n=n, tokens=tokens, features=width, rms=rms, eps=eps)
        self.dense = B.LayerDesc(kind=B.DP_DENSE, in_dtype=B.DP_BF16, n=n, cin=width, cout=vocab, h=tokens, w=1, has_bias=0)
        self.loss = B.LogprobDesc(in_dtype=B.DP_BF16, n=n, tokens=tokens, vocab=vocab, top=0, scale=scale)
        rows, pitch = n * tokens, B.dp_checkpoint_pitch(width)
        byte = dict(dtype=torch.uint8, device=device)
        self.kept = torch.empty(rows * pitch, **byte), torch.empty(rows * pitch // 32, **byte)
        room = max(B.dp_checkpoint_workspace_bytes(self.dense, use) for use in (B.DP_WS_PER_EXAMPLE_GRAD, B.DP_WS_RECOMPUTE))
        self.ws = torch.empty(max(room, B.dp_layer_norm_workspace_bytes(self.norm), B.dp_token_logprobs_workspace_bytes(self.loss), 16), **byte)
        self.g_affine = torch.zeros((n, begins[-1]), **f32)
        self.sqnorm, self.total_sqnorm = torch.empty((2, n), **f32), torch.empty(n, **f32)
        self.one_group = torch.zeros(2, dtype=torch.int32, device=device)
        self.passes = 0                                   # forward and back
        self.logits = None                                # of the forward pass that the block holds
        self._round()

    def _round(self):
        self.projection = self.weights[-1].to(torch.bfloat16)

    def _want(self, name, t, shape, dtype=torch.bfloat16):
        """The calls below take addresses, on the current device: what is behind them has to be what the descriptors say, and there."""
        if tuple(t.shape) != shape or t.dtype is not dtype or t.device != self.theta.device or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} {list(shape)} on {self.theta.device}, not {t.dtype} {list(t.shape)} on {t.device}")
        if t.device.type == "cuda" and t.device.index != torch.cuda.current_device():
            raise ValueError(f"the block is on {self.theta.device}, the current device is {torch.cuda.current_device()}")

    def _want_inputs(self, x, targets, lengths):
        self._want("x", x, (self.n, self.tokens, self.width))
        self._want("targets", targets, (self.n, self.tokens), torch.int32)
        if lengths is not None:
            self._want("lengths", lengths, (self.n,), torch.int32)

    def _shift(self):
        return None if self.rms else self.weights[1]

    def logprobs(self, x, targets, lengths=None):
        """Log probabilities [n, tokens] of targets [n, tokens] int32 after tokens x [n, tokens, width] bf16; zeros for tokens that are not scored."""
        self._want_inputs(x, targets, lengths)
        if x.requires_grad and torch.is_grad_enabled():
            return _Recorded.apply(x, self, targets, lengths)
        with torch.no_grad():
            return self._logprobs(x, targets, lengths)

    def _logits(self, x, lengths):
        normed = torch.empty_like(x)
        B.dp_layer_norm(self.norm, x, self.weights[0], self._shift(), normed, lengths=lengths)
        B.dp_checkpoint_write(normed, *self.kept)
        return (normed.view(-1, self.width) @ self.projection.t()).view(self.n, self.tokens, self.vocab)

    def _logprobs(self, x, targets, lengths):
        self.passes += 1
        self.x, self.targets, self.lengths = x.detach(), targets.clone(), None if lengths is None else lengths.clone()
        self.logits = self._logits(x, lengths)
        f32 = dict(dtype=torch.float32, device=self.theta.device)
        result, self.stats = torch.empty((self.n, self.tokens), **f32), torch.empty((self.n, self.tokens, 2), **f32)
        B.dp_token_logprobs(self.loss, self.logits, targets, result, None, self.stats, None, None, self.ws, lengths=lengths)
        return result

    @torch.no_grad()
    def backward(self, d_logprobs):
        """Derivatives of a sum over examples by logprobs' result -> gradient of its input; the clipped gradients of the parameters go into the accumulator."""
        d_logprobs = d_logprobs.contiguous()
        self._want("d_logprobs", d_logprobs, (self.n, self.tokens), torch.float32)
        if self.logits is None:
            raise RuntimeError("the block holds no forward pass: it has been back over the last one")
        self.passes += 1
        dlogits, self.logits = self.logits, None
        B.dp_token_logprobs_backward(self.loss, dlogits, self.targets, self.stats, d_logprobs, dlogits, self.ws, lengths=self.lengths)
        return self._parameters(self.x, dlogits, self.lengths)

    @torch.no_grad()
    def train(self, x, targets, d_logprobs, lengths=None):
        """Both passes at once, where the tokens' weights are known beforehand -> (log probabilities, gradient of x)."""
        self._want_inputs(x, targets, lengths)
        self._want("d_logprobs", d_logprobs, (self.n, self.tokens), torch.float32)
        self.passes += 1
        self.logits = None
        logits = self._logits(x, lengths)
        result = torch.empty((self.n, self.tokens), dtype=torch.float32, device=self.theta.device)
        B.dp_token_logprobs_backward(self.loss, logits, targets, None, d_logprobs, logits, self.ws, logprobs=result, lengths=lengths)
        return result, self._parameters(x, logits, lengths)

    def _parameters(self, x, dlogits, lengths):
        self.dlogits = dlogits
        dnormed = (dlogits.view(-1, self.vocab) @ self.projection).view(self.n, self.tokens, self.width)
        dx, stride = torch.empty_like(x), self.g_affine.stride(0)
        B.dp_checkpoint_example_grad(self.dense, *self.kept, dlogits, None, None, self.sqnorm[0], self.ws, lengths)
        B.dp_layer_norm_backward(self.norm, x, self.weights[0], dnormed, dx, self.g_affine, None if self.rms else self.g_affine[:, stride // 2:], self.sqnorm[1], self.ws,
                                 lengths=lengths, g_stride=stride)
        B.dp_norms(self.sqnorm, self.one_group, 2, self.n, 1, self.total_sqnorm)
        B.dp_checkpoint_clip_accumulate(self.dense, *self.kept, dlogits, self.total_sqnorm, self.clip_c, self.sums[-1], None, self.ws, lengths)
        B.dp_clip_accumulate(self.g_affine, self.total_sqnorm, self.clip_c, self.n, stride, self.acc, stride)
        return dx

    @torch.no_grad()
    def next_tokens(self, x, top: int = 1):
        """The most likely tokens after x [n, width] bf16, one token an example -> (tokens [n, top] int32, their log probabilities [n, top]).  For serving: leaves
        what a forward pass left alone."""
        self._want("x", x, (self.n, self.width))
        norm = B.NormDesc(in_dtype=B.DP_BF16, n=self.n, tokens=1, features=self.width, rms=self.rms, eps=self.norm.eps)
        normed = torch.empty_like(x)
        B.dp_layer_norm(norm, x, self.weights[0], self._shift(), normed)
        logits = normed @ self.projection.t()
        desc = B.LogprobDesc(in_dtype=B.DP_BF16, n=self.n, tokens=1, vocab=self.vocab, top=top, scale=self.loss.scale)
        ws = torch.empty(max(B.dp_token_logprobs_workspace_bytes(desc), 16), dtype=torch.uint8, device=self.theta.device)
        best = torch.empty((self.n, top), dtype=torch.float32, device=self.theta.device)
        tokens = torch.empty((self.n, top), dtype=torch.int32, device=self.theta.device)
        B.dp_token_logprobs(desc, logits, None, None, None, None, best, tokens, ws)
        return tokens, best

    def step(self, index: int):
        """The optimiser step after total_batch examples: noise, mean, update; the next one's sums begin at zero."""
        bound = self.clip_c if self.clip_total is None else self.clip_total
        B.dp_add_noise_finalize_flat(self.acc, None, self.tensors, self.sigma, bound, self.total_batch, self.seed, index, theta=self.theta,
                                     velocity=self.velocity, lr=self.lr, momentum=self.momentum)
        self.acc.zero_()
        self._round()
