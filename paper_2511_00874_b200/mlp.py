"""The feed-forward half of a transformer layer on block-scaled E4M3 operators, forward and backward.

    r   = x + residual                                   (the stream, kept in x's type)
    y   = rmsnorm(r) * w                                 codes, 1 x 128
    h   = act(y Wg^T) * (y Wu^T)                         codes, 1 x 128; both projections kept as 8-bit checkpoints
    out = h Wd^T                                         (added to r by the next norm)

Every product reads 8-bit codes and every tensor kept for the backward pass but r is 8 bits wide.  The class holds
what a training program holds between steps: the coded weights (row-major for the forward pass, transposed for the
input gradients) and the activations' and gradients' buffers.  The calls only enqueue work on the current stream.

An object is one block of one training step: it takes one number of tokens, allocates every buffer of both passes when it is
built, and each ``forward`` writes the results and checkpoints of the one before it over, so that ``backward`` belongs to the
latest ``forward`` (copy what has to outlive the next call; one object per micro-batch in flight).  ``forward`` always
writes the checkpoints; a program that only generates calls the operators itself and leaves them out of srq_glu_fwd.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from . import binding as B


class GatedMLP:
    def __init__(self, tokens: int, features: int, hidden: int, act: int = B.SILU, dtype: torch.dtype = torch.bfloat16,
                 eps: float = 1e-5, device="cuda"):
        if hidden % B.BLOCK:
            raise ValueError("hidden must be a multiple of 128: the two projections' gradients lie side by side in blocks")
        T, K, F = tokens, features, hidden
        self.shape, self.act, self.eps = (T, K, F), act, eps
        new = lambda r, c, tile=1: B.new_blocks(r, c, tile, device)  # noqa: E731
        e = lambda *s, dt=dtype: torch.empty(s, dtype=dt, device=device)  # noqa: E731
        # weights, 128 x 128 tiles
        self.wg, self.wu, self.wd = new(F, K, B.BLOCK), new(F, K, B.BLOCK), new(K, F, B.BLOCK)
        self.wgu_t, self.wd_t = new(K, 2 * F, B.BLOCK), new(F, K, B.BLOCK)
        self.w: Optional[torch.Tensor] = None
        # forward
        self.y, self.h, self.gate, self.up = new(T, K), new(T, F), new(T, F), new(T, F)
        self.r, self.out, self.rstd = e(T, K), e(T, K), e(T, dt=torch.float32)
        # backward
        self.dout, self.dout_t, self.dgu = new(T, K), new(K, T), new(T, 2 * F)
        self.dg_t, self.du_t, self.h_t, self.y_t = new(F, T), new(F, T), new(F, T), new(K, T)
        self.dh, self.dy, self.dx = e(T, F), e(T, K), e(T, K)
        f = torch.float32
        self.dwg, self.dwu, self.dwd, self.dw = e(F, K, dt=f), e(F, K, dt=f), e(K, F, dt=f), e(K, dt=f)
        self.ws = B.new_workspace(B.srq_rmsnorm_workspace_bytes(T, K), device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    @staticmethod
    def _columns(b: B.Blocks, first: int, n: int) -> B.Blocks:
        return B.Blocks(b.codes[:, first:first + n], b.scale[:, first // B.BLOCK:(first + n + B.BLOCK - 1) // B.BLOCK], b.tile_rows)

    @staticmethod
    def _stream(q: B.QSpec, i: int) -> B.QSpec:
        """q with the thresholds of the i-th stream after its own."""
        return dataclasses.replace(q, tensor_id=q.tensor_id + i)

    def load(self, w: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor, q: B.QSpec = B.BLOCK_RNE) -> None:
        """Codes the weights once per step: wg, wu [hidden, features], wd [features, hidden]; w is the norm's.  Under
        stochastic rounding each weight has a threshold stream of its own: q.tensor_id, + 1 and + 2."""
        _, K, F = self.shape
        self.w = w
        B.srq_quantize_blocks(wg, q, self.wg, self._columns(self.wgu_t, 0, F), self.status)
        B.srq_quantize_blocks(wu, self._stream(q, 1), self.wu, self._columns(self.wgu_t, F, F), self.status)
        B.srq_quantize_blocks(wd, self._stream(q, 2), self.wd, self.wd_t, self.status)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """out = MLP(norm(x + residual)); ``self.r`` holds x + residual."""
        B.srq_rmsnorm_fwd(x, residual, self.w, self.eps, self.y, self.r, self.rstd, device_status=self.status)
        B.srq_glu_fwd(self.y, self.wg, self.wu, self.act, self.h, self.gate, self.up, device_status=self.status)
        B.srq_gemm_blocks(self.h, self.wd, self.out, device_status=self.status)
        return self.out

    def backward(self, dout: torch.Tensor, dr: Optional[torch.Tensor] = None, q: B.QSpec = B.BLOCK_RNE) -> torch.Tensor:
        """Gradient at x (and residual) from the gradients at out and r; the weights' gradients land in ``dwg``,
        ``dwu``, ``dwd`` and ``dw``.  ``q``: how gradients are rounded (block_sr(seed, tensor_id) for stochastic
        rounding; tensor_id .. tensor_id + 3 are used; with a step on the device where the pass is recorded, or every
        replay rounds an element with the same threshold)."""
        F = self.shape[2]
        s = self.status
        B.srq_quantize_blocks(dout, q, self.dout, self.dout_t, s)
        B.srq_gemm_blocks(self.dout, self.wd_t, self.dh, device_status=s)
        B.srq_glu_bwd(self.dh, self.gate, self.up, self.act, self._stream(q, 1), self._columns(self.dgu, 0, F), self._columns(self.dgu, F, F),
                      self.dg_t, self.du_t, self.h_t, s)
        B.srq_gemm_blocks(self.dout_t, self.h_t, self.dwd, device_status=s)
        B.srq_quantize_blocks(self.y, B.BLOCK_RNE, None, self.y_t, s)              # the norm's codes, turned over
        B.srq_gemm_blocks(self.dg_t, self.y_t, self.dwg, device_status=s)
        B.srq_gemm_blocks(self.du_t, self.y_t, self.dwu, device_status=s)
        B.srq_gemm_blocks(self.dgu, self.wgu_t, self.dy, device_status=s)          # dg Wg + du Wu in one contraction
        B.srq_rmsnorm_bwd(self.dy, self.r, self.w, self.rstd, dr, self.dx, self.dw, self.ws)
        return self.dx
