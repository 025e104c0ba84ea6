"""A residual feed-forward block over the embeddings of a node type, as a sequence of library calls.

    h <- x + agg;   h <- h + act(norm(h) W1 + b1) W2 + b2

`agg` is what a layer's relation aggregation yields for the type (RafLayer.H[t], Eq. 1 of the paper), x the embeddings that it
adds to: with such blocks behind its layers a model of this library can be made deep.  The block trains with heta_muon_multi
on its two matrices (`update`), and for inference its first product can run on 8-bit operands.  This module allocates
buffers and orders calls on torch's current stream (the buffers' own: none is given back while a call may still read it); all
arithmetic is in libheta.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple

import torch

from . import binding as hb


class FeedForwardBlock:
    """g: any handle whose workspace the calls may use; blocks that run on streams of their own have handles of their own.
    W1 [d, d_hidden], W2 [d_hidden, d] (fp32 or bf16, like the embeddings); gamma, b1, b2: fp32 vectors or None."""

    def __init__(self, g: hb.Graph, W1: torch.Tensor, W2: torch.Tensor, gamma: Optional[torch.Tensor] = None, b1: Optional[torch.Tensor] = None,
                 b2: Optional[torch.Tensor] = None, act: int = hb.HETA_ACT_GELU, eps: float = 1e-6):
        if W1.shape != W2.shape[::-1]:
            raise ValueError("W1 is [d, d_hidden] and W2 [d_hidden, d]")
        self.g, self.W1, self.W2, self.gamma, self.b1, self.b2, self.act, self.eps = g, W1, W2, gamma, b1, b2, act, eps
        self.m = [torch.zeros(w.shape, dtype=torch.float32, device=w.device) for w in (W1, W2)]
        self.saved: Optional[Dict[str, torch.Tensor]] = None
        self.grads: Dict[str, Optional[torch.Tensor]] = {}

    def forward(self, x: torch.Tensor, agg: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The block's output for the rows x (+ agg), keeping what the backward pass reads."""
        n, d = x.shape
        dev, t, d_hidden = x.device, x.dtype, self.W1.shape[1]
        new = lambda *s: torch.empty(s, dtype=t, device=dev)  # noqa: E731
        h = x if agg is None else new(n, d)
        normed, rstd, pre, hidden, out = new(n, d), torch.empty(n, device=dev), new(n, d_hidden), new(n, d_hidden), new(n, d)
        hb.heta_rms_norm(x, normed, residual=agg, sum=None if agg is None else h, gamma=self.gamma, eps=self.eps, rstd=rstd)
        hb.heta_linear(self.g, normed, self.W1, hidden, bias=self.b1, act=self.act, pre=pre)
        hb.heta_linear(self.g, hidden, self.W2, out, bias=self.b2, residual=h)
        self.saved = {"h": h, "normed": normed, "rstd": rstd, "pre": pre, "hidden": hidden}
        return out

    def backward(self, grad_out: torch.Tensor) -> torch.Tensor:
        """The gradient of x (and of agg), given that of the output; the parameters' gradients are left in `grads`."""
        if self.saved is None:
            raise RuntimeError("forward has not run")
        s, w1, w2 = self.saved, self.W1, self.W2
        vec = lambda v: None if v is None else torch.empty_like(v)  # noqa: E731
        self.grads = {"W1": torch.empty_like(w1), "W2": torch.empty_like(w2), "gamma": vec(self.gamma), "b1": vec(self.b1), "b2": vec(self.b2)}
        g = self.grads
        # the second product's input gradient comes as the gradient at the activation's argument
        grad_pre, grad_normed = torch.empty_like(s["pre"]), torch.empty_like(s["normed"])
        hb.heta_linear_bwd(self.g, s["hidden"], w2, grad_out, grad_in=grad_pre, in_act=self.act, in_pre=s["pre"], grad_W=g["W2"], grad_bias=g["b2"])
        hb.heta_linear_bwd(self.g, s["normed"], w1, grad_pre, grad_in=grad_normed, grad_W=g["W1"], grad_bias=g["b1"])
        grad_x = torch.empty_like(s["h"])
        hb.heta_rms_norm_bwd(self.g, s["h"], s["rstd"], grad_normed, grad_x, gamma=self.gamma, grad_sum=grad_out, grad_gamma=g["gamma"])
        return grad_x

    def muon_items(self) -> List[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]]:
        """This block's part of a heta_muon_multi call (a model's blocks and relation matrices take one call together)."""
        return [(self.W1, self.m[0], self.grads["W1"]), (self.W2, self.m[1], self.grads["W2"])]

    def update(self, lr: float = 0.02, momentum: float = 0.95, weight_decay: float = 0.0) -> None:
        """Orthogonalised momentum on W1 and W2 with the last backward pass's gradients."""
        hb.heta_muon_multi(self.g, self.muon_items(), lr=lr, momentum=momentum, weight_decay=weight_decay)

    def pack(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """W1 as it is now, in 8 bits with a scale per column, for `infer`; to be packed again by whoever changes W1."""
        d, d_hidden = self.W1.shape
        packed, scale = torch.empty((d_hidden, d), dtype=torch.float8_e4m3fn, device=self.W1.device), torch.empty(d_hidden, device=self.W1.device)
        hb.heta_linear_pack_e4m3(self.W1, packed, scale)
        return packed, scale

    def infer(self, x: torch.Tensor, agg: Optional[torch.Tensor] = None, packed: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
              coarse_sums: bool = False) -> torch.Tensor:
        """The output alone.  With `packed` (what `pack` gave; bf16 embeddings) the norm writes its rows in 8 bits and the first product
        reads them and the weights that way; with `coarse_sums` the 8-bit matrix instruction adds, at up to twice the rate (heta_linear)."""
        n, d = x.shape
        dev, t, d_hidden = x.device, x.dtype, self.W1.shape[1]
        h = x if agg is None else torch.empty_like(x)
        sum_ = None if agg is None else h
        hidden, out = torch.empty((n, d_hidden), dtype=t, device=dev), torch.empty((n, d), dtype=t, device=dev)
        if packed is None:
            normed, scales, w, w_scale = torch.empty((n, d), dtype=t, device=dev), None, self.W1, None
        else:
            normed, scales = torch.empty((n, d), dtype=torch.float8_e4m3fn, device=dev), torch.empty(n, device=dev)
            w, w_scale = packed
        hb.heta_rms_norm(x, normed, residual=agg, sum=sum_, gamma=self.gamma, eps=self.eps, scale=scales)
        hb.heta_linear(self.g, normed, w, hidden, bias=self.b1, act=self.act, in_scale=scales, w_scale=w_scale,
                       coarse_sums=coarse_sums and packed is not None)
        hb.heta_linear(self.g, hidden, self.W2, out, bias=self.b2, residual=h)
        return out
