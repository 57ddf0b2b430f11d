"""Trains one private attention block to repeat the token before, which takes its bias table, on synthetic data:

    python examples/private_attention.py [steps]
"""
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2109_12191_amd as dp  # noqa: E402

N, TOKENS, WIDTH, MICRO_STEPS = 64, 32, 64, 4


def main(steps: int = 100, lr: float = 0.5, sigma: float = 0.5):
    block = dp.PrivateAttention(N, TOKENS, WIDTH, heads=4, clip_c=1.0, sigma=sigma, total_batch=N * MICRO_STEPS, lr=lr, momentum=0.9)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for index in range(steps):
        error = torch.zeros((), device="cuda")
        for _ in range(MICRO_STEPS):
            x = torch.randn((N, TOKENS, WIDTH), generator=gen, device="cuda").to(torch.bfloat16)
            lengths = torch.randint(TOKENS // 2, TOKENS + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
            there = (torch.arange(TOKENS, device="cuda")[None] < lengths[:, None])[..., None]
            there[:, 0] = False                       # the first token follows none
            off = (block.forward(x, lengths) - x.roll(1, dims=1)) * there
            error += off.float().square().sum() / (there.sum() * WIDTH)
            block.backward(off / (TOKENS * WIDTH) ** 0.5)
        block.step(index)
        if index % 10 == 0 or index == steps - 1:
            print(f"step {index}: mean squared error {float(error) / MICRO_STEPS:.4f}, {int((block.total_sqnorm > 1.0).sum())} of {N} examples clipped", flush=True)
    return float(error) / MICRO_STEPS


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
