"""The classifier at a model's end, as a sequence of library calls: loss, gradients, update and scores.

    z = h W + b;   loss = mean over the labelled rows of  log sum_j exp z_j - z_label

`h` are the embeddings of the nodes to be classified (RafLayer.H, FeedForwardBlock.forward, the seeds of a MiniBatchTrainer step); the classes are labels
of a node type, or the nodes of a type themselves (which one stands at the other end of a link).  Training never holds the logits in memory
(heta_linear_xent), the update keeps its states in 32 or 8 bits (heta_adamw_multi), and `scores` can run on 8-bit whole numbers.  This module allocates
buffers and orders calls on torch's current stream; all arithmetic is in libheta.
"""
from __future__ import annotations

import itertools
from typing import Callable, Dict, List, Optional, Tuple

import torch

from . import binding as hb

# Seeds of heads that are given none: one each, and far from those of trainers, which count their tensors from their own seed on (0 unless told otherwise).
_SEEDS = itertools.count(1 << 31)


class ClassifierHead:
    """g: any handle whose workspace the calls may use, one for each stream that runs them.  W [d, n_classes] of the embeddings' type (fp32 or bf16),
    bias fp32 [n_classes] or None; state_bits, weight_decay: the update's (the bias has 32-bit states and no decay); seed: of W's 8-bit states, another one for
    each tensor that has such (None: this head's own, 2^31 and one more for each head of the process)."""

    def __init__(self, g: hb.Graph, W: torch.Tensor, bias: Optional[torch.Tensor] = None, state_bits: int = 32, weight_decay: float = 0.0, seed: Optional[int] = None):
        self.g, self.W, self.bias, self.weight_decay, self.seed = g, W, bias, weight_decay, next(_SEEDS) if seed is None else seed
        self.states = [hb.heta_adamw_state(W, state_bits)] + ([] if bias is None else [hb.heta_adamw_state(bias)])
        self.saved: Optional[Dict[str, torch.Tensor]] = None
        self.grads: Dict[str, Optional[torch.Tensor]] = {}
        self.step = 0

    def loss(self, h: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        """The mean loss (a device scalar) of the rows h [n, d] with labels int64 [n] (-1: none), keeping what the backward pass reads; the rows' own losses
        are in saved["loss"]."""
        n, dev = h.shape[0], h.device
        s = {"h": h, "labels": labels, "loss": torch.empty(n, device=dev), "lse": torch.empty(n, device=dev), "mean": torch.empty(2, device=dev)}
        hb.heta_linear_xent(self.g, h, self.W, labels, s["loss"], s["lse"], bias=self.bias, mean=s["mean"])
        self.saved = s
        return s["mean"][0]

    def backward(self, scale: float = 1.0) -> torch.Tensor:
        """The gradient of h, of `scale` times the mean loss; the parameters' are left in `grads`."""
        if self.saved is None:
            raise RuntimeError("loss has not run")
        s = self.saved
        grad_h = torch.empty_like(s["h"], memory_format=torch.contiguous_format)
        self.grads = {"W": torch.empty_like(self.W, memory_format=torch.contiguous_format), "bias": None if self.bias is None else torch.empty_like(self.bias)}
        hb.heta_linear_xent_bwd(self.g, s["h"], self.W, s["labels"], s["lse"], bias=self.bias, scale=scale, mean=s["mean"], grad_in=grad_h, grad_W=self.grads["W"],
                                grad_bias=self.grads["bias"])
        return grad_h

    def loss_grad(self, labels: torch.Tensor) -> Callable[[torch.Tensor], torch.Tensor]:
        """What MiniBatchTrainer.step asks for: embeddings of the seeds with these labels to the loss's gradient there."""
        def of(h: torch.Tensor) -> torch.Tensor:
            self.loss(h, labels)
            return self.backward()
        return of

    def adamw_items(self) -> List[tuple]:
        """This head's part of a heta_adamw_multi call (a model's blocks and heads take one call together)."""
        if not self.grads:
            raise RuntimeError("backward has not run")
        items = [(self.W, self.states[0], self.grads["W"], self.weight_decay, None, self.seed)]
        if self.bias is not None:
            items.append((self.bias, self.states[1], self.grads["bias"]))
        return items

    def update(self, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8) -> None:
        """One AdamW step with the last backward pass's gradients.  Captured into a graph it stays that step: replays do not count (heta_adamw_multi)."""
        hb.heta_adamw_multi(self.adamw_items(), lr=lr, beta1=beta1, beta2=beta2, eps=eps, step=self.step + 1)
        self.step += 1

    def pack(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """W as it is now in 8-bit whole numbers with a scale per class, for `scores`; to be packed again by whoever changes W."""
        d, classes = self.W.shape
        packed, scale = torch.empty((classes, d), dtype=torch.int8, device=self.W.device), torch.empty(classes, device=self.W.device)
        hb.heta_linear_pack_i8(self.W, packed, scale)
        return packed, scale

    def scores(self, h: torch.Tensor, packed: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> torch.Tensor:
        """The logits [n, n_classes] in h's type; with `packed` (what `pack` gave) from rows and weights of 8-bit whole numbers."""
        n, d = h.shape
        out = torch.empty((n, self.W.shape[1]), dtype=h.dtype, device=h.device)
        if packed is None:
            return hb.heta_linear(self.g, h, self.W, out, bias=self.bias)
        rows, scale = torch.empty((n, d), dtype=torch.int8, device=h.device), torch.empty(n, device=h.device)
        hb.heta_linear_rows_i8(h, rows, scale)
        return hb.heta_linear(self.g, rows, packed[0], out, bias=self.bias, in_scale=scale, w_scale=packed[1])
