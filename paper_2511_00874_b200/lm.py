"""A language model's training step on the library's operators, from token ids to updated weights.

    x      = scale * table[ids]                                          embedding
    x, r   = block_l(x, r),  l = 1 .. layers                             mlp.GatedMLP: norm, gated feed-forward block, residual
    logits = norm(x + r) head^T                                          codes, 1 x 128
    loss, dlogits                                                        policy, preference or supervised; the gradient takes the logits' place
    backward through all of it
    AdamW on every weight (bfloat16, stochastically rounded; moments in 8 or 32 bits), and the new weights' codes

The model mixes nothing between tokens: it is the part of a transformer that this library has operators for, which is where its weights
are.  Like GatedMLP it takes one number of tokens and allocates everything when it is built; calls only enqueue work on the current
stream, so that a whole step can be recorded in a CUDA graph (``ids`` and targets in buffers that stay; the number of the step and the
learning rate live on the device).
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from . import binding as B
from .mlp import GatedMLP


class TokenModel:
    def __init__(self, tokens: int, vocab: int, features: int, hidden: int, layers: int, act: int = B.SILU, state_bits: int = 8,
                 embedding_scale: float = 1.0, eps: float = 1e-5, seed: int = 0, device="cuda"):
        T, V, K = tokens, vocab, features
        dt = torch.bfloat16
        self.shape, self.scale, self.eps, self.seed = (T, V, K), embedding_scale, eps, seed
        new = lambda r, c, tile=1: B.new_blocks(r, c, tile, device)  # noqa: E731
        e = lambda *s, d=dt: torch.empty(s, dtype=d, device=device)  # noqa: E731
        self.blocks = [GatedMLP(T, K, hidden, act, dt, eps, device) for _ in range(layers)]
        # weights: matrices, then norms (which do not decay)
        self.table, self.head = e(V, K), e(V, K)
        self.layers = [(e(hidden, K), e(hidden, K), e(K, hidden)) for _ in range(layers)]
        self.norms = [e(K) for _ in range(layers + 1)]
        # forward and backward
        self.x, self.y, self.r, self.rstd = e(T, K), new(T, K), e(T, K), e(T, d=torch.float32)
        self.head_codes, self.head_codes_t = new(V, K, B.BLOCK), new(K, V, B.BLOCK)
        self.logits = torch.empty((T, -(-V // 8) * 8), dtype=dt, device=device)[:, :V]
        self.dl, self.dl_t, self.y_t = new(T, V), new(V, T), new(K, T)
        self.dy, self.dx = e(T, K), e(T, K)
        f = torch.float32
        self.dtable, self.dhead, self.dnorm = e(V, K, d=f), e(V, K, d=f), e(K, d=f)
        self.logp, self.lse, self.row_loss, self.loss = e(T, d=f), e(T, d=f), e(T, d=f), e(1, d=f)
        self.ws = B.new_workspace(max(B.srq_embedding_workspace_bytes(T, V, K), B.srq_rmsnorm_workspace_bytes(T, K), B.srq_preference_workspace_bytes(T)), device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)      # what any part of a step reports, the layers included
        for b in self.blocks:
            b.status = self.status
        # update
        weights = [self.table, self.head] + [w for layer in self.layers for w in layer]
        grads = [self.dtable, self.dhead] + [g for b in self.blocks for g in (b.dwg, b.dwu, b.dwd)]
        norm_grads = [b.dw for b in self.blocks] + [self.dnorm]
        tensors = lambda ws, gs: B.AdamTensors([B.AdamTensor(w, g, *B.new_adam_state(w, state_bits)) for w, g in zip(ws, gs)])  # noqa: E731
        self.decaying, self.plain = tensors(weights, grads), tensors(self.norms, norm_grads)
        self.step, self.lr = torch.zeros(1, dtype=torch.int64, device=device), torch.zeros(1, device=device)
        self.next_step = torch.zeros_like(self.step)

    def initialise(self, std: float = 0.02) -> None:
        """Weights from N(0, std^2), norms one."""
        g = torch.Generator(device=self.table.device).manual_seed(self.seed)
        for w in [self.table, self.head] + [w for layer in self.layers for w in layer]:
            w.copy_(torch.randn(w.shape, generator=g, device=w.device) * std)
        for w in self.norms:
            w.fill_(1.0)
        self.load()

    def load(self) -> None:
        """Codes of the weights as they are."""
        for b, w, layer in zip(self.blocks, self.norms, self.layers):
            b.load(w, *layer)
        B.srq_quantize_blocks(self.head, B.BLOCK_RNE, self.head_codes, self.head_codes_t, self.status)

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        """Logits of the tokens (ids below zero: padding, a row of zeros into the first layer)."""
        s = self.status
        B.srq_embedding_fwd(self.table, ids, self.x, self.scale, s)
        x, r = self.x, None
        for b in self.blocks:
            x, r = b.forward(x, r), b.r
        B.srq_rmsnorm_fwd(x, r, self.norms[-1], self.eps, self.y, self.r, self.rstd, device_status=s)
        B.srq_gemm_blocks(self.y, self.head_codes, self.logits, device_status=s)
        return self.logits

    def supervised(self, targets: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
        """Minus the weighted sum of the targets' log-probabilities; targets below zero and weights of zero do not count.  Logits become
        gradients."""
        if weight.shape != self.row_loss.shape:
            raise ValueError(f"weight must hold {len(self.row_loss)} values, got {tuple(weight.shape)}")
        targets = torch.where(weight != 0, targets, -1)
        B.srq_logprob_fwd(self.logits, targets, self.logp, self.lse, device_status=self.status)
        torch.mul(weight, -1.0, out=self.row_loss)
        B.srq_logprob_bwd(self.logits, targets, self.lse, self.row_loss, self.logits, device_status=self.status)
        self.row_loss.mul_(self.logp)
        torch.sum(self.row_loss, 0, keepdim=True, out=self.loss)
        return self.loss

    def policy(self, targets: torch.Tensor, logp_old: torch.Tensor, advantage: torch.Tensor, weight: torch.Tensor,
               logp_ref: Optional[torch.Tensor] = None, **kw) -> torch.Tensor:
        """Clipped policy loss (srq_policy_loss); logits become gradients."""
        B.srq_policy_loss(self.logits, targets, logp_old, advantage, weight, logp_ref, self.row_loss, self.loss, self.logp, self.logits,
                          device_status=self.status, **kw)
        return self.loss

    def preference(self, targets: torch.Tensor, logp_ref: torch.Tensor, offsets: torch.Tensor, pair_loss: torch.Tensor, **kw) -> torch.Tensor:
        """Preference loss over pairs of answers (srq_preference_loss); logits become gradients, zero for tokens that belong to no answer."""
        B.srq_preference_loss(self.logits, targets, logp_ref, offsets, pair_loss, self.loss, self.logp, self.logits, ws=self.ws,
                              device_status=self.status, clear_rest=True, **kw)
        return self.loss

    def backward(self, ids: torch.Tensor, q: B.QSpec = B.BLOCK_RNE) -> None:
        """Gradients of every weight from the gradient at the logits; ``q``: how gradients are rounded, with tensor_id ..
        tensor_id + 4 * (layers + 1) under stochastic rounding, and thresholds of their own for every step (``self.step``, read on
        the device, so that replays of a recorded step draw new ones too)."""
        s = self.status
        if q.round == B.SR and q.step is None:
            q = dataclasses.replace(q, step=self.step)
        at = lambda i: GatedMLP._stream(q, 4 * i)  # noqa: E731
        B.srq_quantize_blocks(self.logits, q, self.dl, self.dl_t, s)
        B.srq_quantize_blocks(self.y, B.BLOCK_RNE, None, self.y_t, s)
        B.srq_gemm_blocks(self.dl_t, self.y_t, self.dhead, device_status=s)
        B.srq_gemm_blocks(self.dl, self.head_codes_t, self.dy, device_status=s)
        B.srq_rmsnorm_bwd(self.dy, self.r, self.norms[-1], self.rstd, None, self.dx, self.dnorm, self.ws)
        d = self.dx
        for i, b in reversed(list(enumerate(self.blocks))):
            d = b.backward(d, d, at(i + 1))
        B.srq_embedding_bwd(d, ids, self.dtable, self.scale, ws=self.ws, device_status=s)

    def update(self, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, weight_decay: float = 0.1,
               grad_scale: Optional[torch.Tensor] = None) -> None:
        """AdamW step number ``self.step`` + 1 with the learning rate in ``self.lr``, and the new weights' codes.  A step that is refused
        because the learning rate or ``grad_scale`` is not finite changes nothing and is not counted: ``self.step`` stays."""
        torch.add(self.step, 1, out=self.next_step)
        kw = dict(lr=0.0, beta1=beta1, beta2=beta2, eps=eps, seed=self.seed, lr_device=self.lr, step_device=self.next_step, grad_scale=grad_scale,
                  device_status=self.status)
        B.srq_adamw_step(self.decaying, weight_decay=weight_decay, tensor_id=1 << 16, **kw)
        B.srq_adamw_step(self.plain, weight_decay=0.0, tensor_id=(1 << 16) + len(self.decaying), **kw)
        done = self.lr.isfinite()
        if grad_scale is not None:
            done &= grad_scale.view(-1)[:1].isfinite()
        self.step.add_(done)
        self.load()
