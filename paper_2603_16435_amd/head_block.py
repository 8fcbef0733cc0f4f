"""The block in front of the LM head, trained together with it: final layer norm, a projection on 8-bit operands, then the policy loss.

    y = layer_norm(x) gamma + beta,   hidden = pack(y) W^T,   loss = policy loss of (hidden, LM head)

What the forward pass keeps for the backward pass is in 8 bits: x for the norm, y for the weight gradient (a byte and 1/128 a value each instead of two or
four), so that x may be overwritten.  Every step runs in the HIP library; this module only holds the pieces together."""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding


@dataclass
class HeadKept:
    """What the backward pass needs of a forward pass."""
    stats: torch.Tensor                      # [R, 2] float32: mean, reciprocal standard deviation
    x: binding.F8Rows
    y: binding.F8Rows

    def bytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.stats, self.x.codes, self.x.scales, self.y.codes, self.y.scales))


@dataclass
class HeadGrads:
    dx: torch.Tensor                         # [R, H] in the dtype of x
    dgamma: torch.Tensor                     # float32, as the two below
    dbeta: torch.Tensor
    dweight: torch.Tensor                    # [N, H]
    dlm_head: torch.Tensor                   # [V, N]


class HeadBlock:
    """gamma, beta [H], weight [N, H]: float32 parameters of the norm and the projection; lm_head [V, N] in the dtype of the activations.
    After the parameters changed, `pack()` brings the packed weight up to date."""

    def __init__(self, gamma, beta, weight, lm_head, eps=1e-5, fmt="e4m3", grad_fmt="e5m2"):
        self.gamma, self.beta, self.weight, self.lm_head = gamma, beta, weight, lm_head
        self.eps, self.fmt, self.grad_fmt = eps, fmt, grad_fmt
        self.pack()

    def pack(self):
        self.packed = binding.rl_f8_pack_weight(self.weight, self.fmt)

    def hidden(self, x):
        """The LM head's input for x [R, H], nothing kept: scoring, or a decode step."""
        y = binding.rl_layer_norm_forward(x, self.gamma, self.beta, self.eps, want_stats=False)[0]
        return binding.rl_f8_linear_forward(y, self.packed, self.fmt, keep=False)[0]

    def forward(self, x, overwrite=False):
        """(hidden [R, N], kept).  overwrite: the norm's output takes the place of x."""
        y, stats, kept_x = binding.rl_layer_norm_forward(x, self.gamma, self.beta, self.eps, checkpoint=self.fmt, out=x if overwrite else None)
        hidden, kept_y = binding.rl_f8_linear_forward(y, self.packed, self.fmt)
        return hidden, HeadKept(stats, kept_x, kept_y)

    def backward(self, d_hidden, kept: HeadKept):
        """(dx, dgamma, dbeta, dweight) from the gradient of `hidden`."""
        dy, dweight = binding.rl_f8_linear_backward(d_hidden, kept.y, self.packed, self.grad_fmt)
        dx, dgamma, dbeta = binding.rl_layer_norm_backward(dy, kept.x, kept.stats, self.gamma, out=dy)
        return dx, dgamma, dbeta, dweight

    def policy_step(self, objective, x, token_ids, mask, cu_seqlens, group_idx, rewards, old_logprob, ref_logprob, log_z=None, P=None, overwrite=False, **options):
        """One pass over a batch of rollouts whose last block left x [R, H]: (LossResult, HeadGrads).  options: those of rl_policy_loss_fwd_bwd."""
        hidden, kept = self.forward(x, overwrite)
        res = binding.rl_policy_loss_fwd_bwd(objective, hidden, self.lm_head, token_ids, mask, cu_seqlens, group_idx, rewards, old_logprob, ref_logprob, log_z, P, **options)
        dx, dgamma, dbeta, dweight = self.backward(res.d_hidden, kept)
        return res, HeadGrads(dx, dgamma, dbeta, dweight, res.d_weight)
