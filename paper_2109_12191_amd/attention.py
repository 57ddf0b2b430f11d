"""A self-attention block under a learned relative position bias, trained privately: a small example of the token operators together.

Per micro-step of `n` examples of up to `tokens` tokens:
    forward    dp_checkpoint_write of the block's input, q, k and v of it, dp_bias_softmax of their scores, dp_checkpoint_write of what the
               probabilities make of v, and its projection.  Kept for the backward pass: two 8-bit checkpoints, q, k, v, probabilities
    backward   dp_bias_softmax_backward (the scores' gradient, and each example's gradient of the bias table with its squared norm),
               dp_checkpoint_example_grad of the four projections (squared norms alone), dp_norms, then dp_checkpoint_clip_accumulate and
               dp_clip_accumulate into the flat accumulator
and per optimiser step dp_add_noise_finalize_flat with the SGD update.  The projections themselves and the products of attention are the
framework's user's own matrix products, here torch's.

An example's gradient is that of its checkpoints' values, for the norm and for the clipped sum alike, so that what the checkpoints round away does
not matter to the bound: no more than clip_c of an example gets into the sum, to within the norms' own rounding (dp_checkpoint_example_grad).

forward's result carries a graph where its input requires a gradient: autograd's pass over it is `backward`, with the clipped sums of the weights that
belong to it, and gives the input's gradient.  Elsewhere `backward` is called.  The block holds the values of one forward pass, its lengths among
them, for one such pass back.

examples/private_attention.py trains one on synthetic data.
"""
from __future__ import annotations

import torch

from . import binding as B


class _Recorded(torch.autograd.Function):
    """A forward pass that autograd knows of as a whole: its own products and softmax are not for it to see one by one."""

    @staticmethod
    def forward(ctx, x, block, lengths):
        y = block._forward(x, lengths)
        ctx.block, ctx.passes = block, block.passes
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        if ctx.block.passes != ctx.passes:
            raise RuntimeError("the block no longer holds this forward pass: there was another one, or a pass back over it")
        return ctx.block.backward(dy), None, None


class PrivateAttention:
    """Weights [q; k; v] (three of [width, width], one after the other), the output's [width, width] and the bias table [buckets, heads], fp32 in
    one vector `theta`; activations are bf16.  Tokens beyond an example's length (int32 `lengths`, None: all there) count for nothing,
    but the activations and gradients there have to be finite.

    The noise of a tensor is a function of seed, step and its number, from first_tensor on: blocks of one model and one seed need numbers of their own (the next block's
    first_tensor is this one's next_tensor), or two tensors get the same noise, which a difference takes out again.

    clip_c bounds what an example adds to this block.  A model of several blocks releases all their updates, so an example's part in what is released is bounded by the square
    root of the sum of the blocks' clip_c squared (dp_group_clip_bounds shares a bound out): that is every block's clip_total, which its noise has sigma times of.  None:
    the block is the whole model."""

    def __init__(self, n: int, tokens: int, width: int, heads: int, clip_c: float, sigma: float, total_batch: int, lr: float = 0.0, momentum: float = 0.0,
                 seed: int = 0, buckets: int = 32, max_distance: int = 128, bidirectional: bool = True, causal: bool = False, device: str = "cuda",
                 first_tensor: int = 0, clip_total: float | None = None):
        if width % heads or width // heads % 2:
            raise ValueError(f"{width} features cannot be shared by {heads} heads")
        if not 0 <= first_tensor < (1 << 32) - 5:
            raise ValueError(f"first_tensor {first_tensor} and those behind it are not numbers of 32 bits")
        self.n, self.tokens, self.width, self.heads, self.head = n, tokens, width, heads, width // heads
        if clip_total is not None and not clip_total >= clip_c * (1.0 - 2.0 ** -23):          # (bounds are fp32 to the library)
            raise ValueError(f"clip_total {clip_total} does not cover this block's own clip_c {clip_c}")
        self.clip_total = clip_total
        self.clip_c, self.sigma, self.total_batch, self.lr, self.momentum, self.seed = clip_c, sigma, total_batch, lr, momentum, seed
        self.buckets, self.device = buckets, device
        sizes = [width * width] * 4 + [buckets * heads]
        begins = [0]
        for size in sizes:
            begins.append(begins[-1] + (size + 3) // 4 * 4)
        f32 = dict(dtype=torch.float32, device=device)
        self.theta, self.acc, self.velocity = torch.zeros(begins[-1], **f32), torch.zeros(begins[-1], **f32), torch.zeros(begins[-1], **f32)
        self.tensors = B.TensorTable(begins[:-1], sizes, range(first_tensor, first_tensor + 5))
        self.next_tensor = first_tensor + 5               # the first number that is none of this block's
        view = lambda flat: [flat[b:b + s].view(*shape) for b, s, shape in zip(begins, sizes, [(width, width)] * 4 + [(buckets, heads)])]
        self.weights, self.sums = view(self.theta), view(self.acc)
        gen = torch.Generator(device=device).manual_seed(seed)
        for w in self.weights[:4]:
            w.normal_(0.0, width ** -0.5, generator=gen)
        self.dense = B.LayerDesc(kind=B.DP_DENSE, in_dtype=B.DP_BF16, n=n, cin=width, cout=width, h=tokens, w=1, has_bias=0)
        self.bias = B.BiasDesc(in_dtype=B.DP_BF16, n=n, heads=heads, queries=tokens, keys=tokens, buckets=buckets, max_distance=max_distance,
                               bidirectional=bidirectional, causal=causal, query_offset=0, scale=self.head ** -0.5)
        # decoding: one query an example, its last token, against a cache of `tokens` keys
        self.last = B.BiasDesc(in_dtype=B.DP_BF16, n=n, heads=heads, queries=1, keys=tokens, buckets=buckets, max_distance=max_distance,
                               bidirectional=bidirectional, causal=causal, query_offset=B.DP_QUERIES_AT_END, scale=self.head ** -0.5)
        rows, pitch = n * tokens, B.dp_checkpoint_pitch(width)
        byte = dict(dtype=torch.uint8, device=device)
        self.inputs, self.mixed = [(torch.empty(rows * pitch, **byte), torch.empty(rows * pitch // 32, **byte)) for _ in range(2)]
        room = max(B.dp_checkpoint_workspace_bytes(self.dense, use) for use in (B.DP_WS_PER_EXAMPLE_GRAD, B.DP_WS_RECOMPUTE))
        self.ws = torch.empty(max(room, B.dp_bias_workspace_bytes(self.bias), 16), **byte)
        self.g_table = torch.zeros((n, (buckets * heads + 3) // 4 * 4), **f32)
        self.sqnorm, self.total_sqnorm = torch.empty((5, n), **f32), torch.empty(n, **f32)
        self.one_group = torch.zeros(5, dtype=torch.int32, device=device)
        self.passes = 0                                   # forward and back
        self._round()

    def _round(self):
        self.qkv_weight = torch.cat([w.to(torch.bfloat16) for w in self.weights[:3]])        # [3 width, width]
        self.o_weight = self.weights[3].to(torch.bfloat16)

    def _want(self, name, t, shape, dtype=torch.bfloat16):
        """The calls below take addresses, on the current device: what is behind them has to be what the descriptors say, and there."""
        if tuple(t.shape) != shape or t.dtype is not dtype or t.device != self.theta.device or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} {list(shape)} on {self.theta.device}, not {t.dtype} {list(t.shape)} on {t.device}")
        if t.device.type == "cuda" and t.device.index != torch.cuda.current_device():
            raise ValueError(f"the block is on {self.theta.device}, the current device is {torch.cuda.current_device()}")

    def _want_lengths(self, lengths):
        if lengths is not None:
            self._want("lengths", lengths, (self.n,), torch.int32)

    def _heads(self, x):
        return x.view(self.n, -1, self.heads, self.head).transpose(1, 2).contiguous()         # [n, heads, tokens, head]

    def _tokens(self, x):
        return x.transpose(1, 2).reshape(self.n, -1, self.width)                               # and back

    def forward(self, x, lengths=None):
        """x [n, tokens, width] bf16 -> what the block makes of it, alike."""
        self._want("x", x, (self.n, self.tokens, self.width))
        self._want_lengths(lengths)
        if x.requires_grad and torch.is_grad_enabled():
            return _Recorded.apply(x, self, lengths)
        with torch.no_grad():
            return self._forward(x, lengths)

    def _forward(self, x, lengths):
        self.passes += 1
        self.lengths = None if lengths is None else lengths.clone()
        B.dp_checkpoint_write(x, *self.inputs)
        self.q, self.k, self.v = (self._heads(part) for part in (x @ self.qkv_weight.t()).chunk(3, dim=-1))
        scores = self.q @ self.k.transpose(2, 3).contiguous()
        self.probs = torch.empty_like(scores)
        B.dp_bias_softmax(self.bias, scores, self.weights[4], self.probs, lengths, lengths)
        mixed = self._tokens(self.probs @ self.v)
        B.dp_checkpoint_write(mixed, *self.mixed)
        return mixed @ self.o_weight.t()

    @torch.no_grad()
    def attend_last(self, q, k, v, lengths=None):
        """One token an example against a cache: q [n, width], k and v [n, heads, tokens, head], `lengths` keys of which are there, the query's
        own the last -> [n, width].  For serving: the result carries no graph."""
        self._want("q", q, (self.n, self.width))
        for name, t in (("k", k), ("v", v)):
            self._want(name, t, (self.n, self.heads, self.tokens, self.head))
        self._want_lengths(lengths)
        scores = self._heads(q.view(self.n, 1, self.width)) @ k.transpose(2, 3).contiguous()
        probs = torch.empty_like(scores)
        B.dp_bias_softmax(self.last, scores, self.weights[4], probs, None, lengths)
        return self._tokens(probs @ v).view(self.n, self.width) @ self.o_weight.t()

    @torch.no_grad()
    def backward(self, dy):
        """Gradient of forward's result, per example (of a sum over examples, not of a mean) -> gradient of its input; the clipped gradients of
        the weights go into the accumulator."""
        dy = dy.contiguous()
        self._want("dy", dy, (self.n, self.tokens, self.width))
        self.passes += 1
        dmixed = self._heads(dy @ self.o_weight)
        self.dprobs = dmixed @ self.v.transpose(2, 3).contiguous()
        dv = self.probs.transpose(2, 3).contiguous() @ dmixed
        dscores = torch.empty_like(self.probs)
        B.dp_bias_softmax_backward(self.bias, self.probs, self.dprobs, dscores, self.g_table, self.sqnorm[4], self.ws, self.lengths, self.lengths,
                                   g_stride=self.g_table.stride(0))
        dq, dk = dscores @ self.k, dscores.transpose(2, 3).contiguous() @ self.q
        self.grads = [self._tokens(g) for g in (dq, dk, dv)] + [dy]
        for i, g in enumerate(self.grads):
            B.dp_checkpoint_example_grad(self.dense, *self._checkpoint(i), g, None, None, self.sqnorm[i], self.ws, self.lengths)
        B.dp_norms(self.sqnorm, self.one_group, 5, self.n, 1, self.total_sqnorm)
        for i, g in enumerate(self.grads):
            B.dp_checkpoint_clip_accumulate(self.dense, *self._checkpoint(i), g, self.total_sqnorm, self.clip_c, self.sums[i], None, self.ws, self.lengths)
        B.dp_clip_accumulate(self.g_table, self.total_sqnorm, self.clip_c, self.n, self.buckets * self.heads, self.sums[4], self.g_table.stride(0))
        return torch.cat(self.grads[:3], dim=-1) @ self.qkv_weight

    def _checkpoint(self, i):
        return self.inputs if i < 3 else self.mixed

    def step(self, index: int):
        """The optimiser step after total_batch examples: noise, mean, update; the next one's sums begin at zero."""
        bound = self.clip_c if self.clip_total is None else self.clip_total
        B.dp_add_noise_finalize_flat(self.acc, None, self.tensors, self.sigma, bound, self.total_batch, self.seed, index, theta=self.theta,
                                     velocity=self.velocity, lr=self.lr, momentum=self.momentum)
        self.acc.zero_()
        self._round()
