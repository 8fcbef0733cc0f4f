"""Trains the block in front of the LM head (layer norm, 8-bit projection) and the LM head itself on one batch of rollouts with the flow-balance objective.

    python examples/train_head_block.py [--steps 20] [--hidden 1024] [--inner 768] [--vocab 8000]

The rollouts are synthetic (paper_2603_16435_amd/synth.py); their old and reference log-probs are scored with the block's own starting parameters."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_16435_amd import binding, synth          # noqa: E402
from paper_2603_16435_amd.head_block import HeadBlock    # noqa: E402


def make(hidden=1024, inner=768, vocab=8000, dtype=torch.bfloat16, seed=5):
    """(block, batch, x, old log-probs): a block over x [R, hidden] that feeds an LM head [vocab, inner]."""
    b = synth.make_rollouts(synth.RolloutConfig("head", 4, 4, 16, 96, hidden, vocab, "bf16", 0.5, seed=seed), "cuda", "padded")
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    block = HeadBlock(1 + 0.1 * n(hidden), 0.1 * n(hidden), n(inner, hidden) / hidden ** 0.5, (0.02 * n(vocab, inner)).to(dtype))
    x = b.hidden.to(dtype)
    old, _ = binding.rl_token_logprob(block.hidden(x), block.lm_head, b.token_ids, b.mask, b.cu_seqlens)
    return block, b, x, old


def train(block, b, x, old, steps, lr=2e-3):
    """Plain gradient descent, every parameter's step scaled by its own gradient's norm; the losses on the way."""
    losses = []
    for _ in range(steps):
        res, g = block.policy_step("flow", x, b.token_ids, b.mask, b.cu_seqlens, b.group_idx, b.rewards, old, old, b.log_z, P=b.log_z.numel(), beta=1.0)
        losses.append(res.loss)
        for p, d in ((block.gamma, g.dgamma), (block.beta, g.dbeta), (block.weight, g.dweight), (block.lm_head, g.dlm_head)):
            p.sub_((lr * p.float().norm() / d.norm().clamp_min(1e-20) * d).to(p.dtype))
        block.pack()
    return torch.stack(losses).flatten().tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, value in (("steps", 20), ("hidden", 1024), ("inner", 768), ("vocab", 8000)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    block, b, x, old = make(a.hidden, a.inner, a.vocab)
    _, kept = block.forward(x)
    print(f"{x.shape[0]} rows of {a.hidden}: kept for the backward pass {kept.bytes() / 1e6:.2f} MB, {2 * x.numel() * x.element_size() / 1e6:.2f} MB as they are")
    for i, loss in enumerate(train(block, b, x, old, a.steps)):
        print(f"step {i}: loss {loss:.6f}")
