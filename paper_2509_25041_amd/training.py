"""Backward pass of a GraceMoELayer step, on buffers that are allocated once."""
from __future__ import annotations

from typing import List, Optional, Tuple

import torch

from .binding import (grace_combine_backward, grace_expert_ffn_backward, grace_ffn_backward_workspace_bytes, grace_permute_backward,
                      grace_route_backward, grace_shared_ffn_backward)
from .layer import GraceMoELayer


class GraceMoEBackward:
    """Gradients of one layer: combine -> gate, experts' FFN [-> shared experts' FFN] -> dispatch, each a call of the library.

    `backward` follows a `forward` of the layer (eager or replayed) and uses what that step left in the layer's buffers: the
    dispatch order, the dispatched rows, the experts' results and the gate weights; the experts' hidden activations are computed again.
    On a rank that does not host every instance the gradients are those of the rank's own rows, as the layer's output is: `dx` and `dlogits`
    are to be summed over the ranks (the shared experts' part of `dx` is in every rank's).  `dw` is of the rank's instances: an expert that is on
    several ranks has the sum of its instances' gradients, which has to be made (an all-reduce among the ranks that host it) before
    grace_grad_norm, grace_clip_grads and the optimizer; otherwise its replicas drift apart, and the norm of the parts is not that of their sum.

    Results are in buffers of this object, overwritten by the next step: `dx` [T,d] (through the experts and the shared experts),
    `dlogits` [T,E] (the gate's own weights are the caller's), and the weights' gradients `dw` (gate, up, down [S,...]) and `dshared`
    ([n_shared,...], None without shared experts).  The pass enqueues only kernels on torch's current stream and can be captured
    in a HIP graph after one eager call.
    """

    def __init__(self, layer: GraceMoELayer):
        self.layer = layer
        T, k, d, f, S = layer.T, layer.k, layer.d, layer.f, layer.w[0].shape[0]
        device = layer.xp.device
        self.dy, self.dxp = torch.zeros_like(layer.xp), torch.zeros_like(layer.xp)
        self.dweight = torch.empty((T, k), dtype=torch.float32, device=device)
        self.dlogits = torch.empty((T, layer.table.E), dtype=torch.float32, device=device)
        self.dx = torch.empty((T, d), dtype=layer.xp.dtype, device=device)
        self.dw = tuple(torch.zeros_like(w) for w in layer.w)
        self.dshared: Optional[Tuple[torch.Tensor, ...]] = None
        need = grace_ffn_backward_workspace_bytes(T * k, d, f, 0, layer.dt) if S else 0
        if layer.n_shared:
            self.dshared = tuple(torch.empty_like(w) for w in layer.shared)
            self.dx_shared = torch.empty_like(self.dx)
            need = max(need, grace_ffn_backward_workspace_bytes(T, d, f, layer.n_shared, layer.dt))
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)

    def gradients(self) -> List[torch.Tensor]:
        """The weights' gradients, for grace_clip_grad_norm and the optimizer (where experts are replicated, after their instances' sums)."""
        return list(self.dw) + list(self.dshared or ())

    def backward(self, dout: torch.Tensor, logits: torch.Tensor, x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """(dx, dlogits) from the gradient of the layer's output; logits and x are the forward step's."""
        layer = self.layer
        expert, weight = layer.route_out[:2]
        pos, _, inst_off, rank_off = layer.perm_out[:4]
        share = (None, 0) if layer.hosts_all else (rank_off, layer.local_rank)
        grace_combine_backward(dout, layer.y, pos, weight, *share, self.dy, self.dweight)
        grace_route_backward(logits, expert, weight, self.dweight, layer.renorm, self.dlogits)
        if layer.w[0].shape[0]:
            grace_expert_ffn_backward(layer.table, layer.local_rank, layer.xp, self.dy, inst_off, layer.T, layer.k, *layer.w, self.dxp, self.dw,
                                      self.ws)
        if layer.n_shared:
            grace_shared_ffn_backward(x, dout, *layer.shared, self.dx_shared, self.dshared, self.ws)
        grace_permute_backward(self.dxp, pos, layer.k, self.dx_shared if layer.n_shared else None, *share, self.dx)
        return self.dx, self.dlogits
