"""Stacked refinement of sketches (paper Sec. 3.3): a layer takes the sketch state X~ [B, H, P, d] of every user
and attends to the user's history X again, with queries of the user's own state:

    A = softmax over the prototypes of scale (X~ W_Q) (X W_K)^T
    X1 = LN(X~ + A X),   X~' = LN(X1 + FFN(X1)),   FFN(u) = (swish(u W_1) * (u W_g)) W_2

Heads are independent copies and share a layer's weights.  Everything is differentiable, in the
history, the state and the weights.
"""
from __future__ import annotations

import math
from typing import Iterable, NamedTuple, Optional

import torch

from . import binding as b


class RefineLayer(NamedTuple):
    """Weights of one layer, of the history's type, as ``sa_linear`` takes them ([outputs, inputs])."""
    w_q: torch.Tensor       # [d, d]
    w_k: torch.Tensor       # [d, d]
    norm1_w: torch.Tensor   # [d]
    norm1_b: torch.Tensor
    w_in: torch.Tensor      # [2 F, d]: the rows of W_1, then those of W_g
    w_out: torch.Tensor     # [d, F]
    norm2_w: torch.Tensor
    norm2_b: torch.Tensor


def random_layer(d: int, F: int, dtype=torch.bfloat16, device="cuda", generator=None) -> RefineLayer:
    def matrix(rows, cols):
        return (torch.randn((rows, cols), generator=generator, device=device) / math.sqrt(cols)).to(dtype)

    ones, zeros = torch.ones(d, dtype=dtype, device=device), torch.zeros(d, dtype=dtype, device=device)
    return RefineLayer(matrix(d, d), matrix(d, d), ones, zeros, matrix(2 * F, d), matrix(d, F), ones.clone(),
                       zeros.clone())


def sa_refine_layer(state: torch.Tensor, X: torch.Tensor, cu_seqlens: torch.Tensor, layer: RefineLayer,
                    scale: Optional[float] = None, eps: float = 1e-5) -> torch.Tensor:
    """The next state [B, H, P, d] of X's type for the state (of the same type) and the histories X [N, H, d]."""
    keys = b.sa_linear(X, layer.w_k)
    queries = b.sa_linear(state, layer.w_q)
    aggregated = b.sa_sketch(keys, X, cu_seqlens, queries, scale)  # fp32
    x1 = b.sa_layer_norm(aggregated, layer.norm1_w, layer.norm1_b, residual=state, eps=eps, dtype=X.dtype)
    hidden = b.sa_linear(x1, layer.w_in, activation="swiglu")
    return b.sa_layer_norm(b.sa_linear(hidden, layer.w_out, residual=x1), layer.norm2_w, layer.norm2_b, eps=eps)


def sa_refine(sketch: torch.Tensor, X: torch.Tensor, cu_seqlens: torch.Tensor, layers: Iterable[RefineLayer],
              scale: Optional[float] = None, eps: float = 1e-5) -> torch.Tensor:
    """The state after all layers, [B, H, P, d] of X's type, from the first sketch (``sa_sketch``'s, fp32)."""
    state = sketch.to(X.dtype)
    for layer in layers:
        state = sa_refine_layer(state, X, cu_seqlens, layer, scale, eps)
    return state
