"""One mixture-of-experts layer around the routing step, forward and backward.

    n = norm(x)   logits = n Wr^T   ids, w = gate(logits)   send = route(n, ids)   o = experts(send)
    y = combine(o, w)   out = x + dropout(y)

Plumbing only, as in `router`: torch allocates the buffers once and multiplies by the router's weights (a plain library
product); everything else is one C-ABI call each, enqueued on the current torch stream.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as cb
from .router import RouteStep


class MoELayer:
    """Parameters, their gradients and the buffers of one layer for T tokens of width H over the experts of `layout`.

    slot_expert: expert of every slot (-1 = empty), as given to the layout.  gate: "softmax" or "sigmoid".
    Parameters: gamma, beta float32 [H]; w_router bfloat16 [E, H]; w_gate_up [E, 2F, H]; w_down [E, H, F].
    """

    def __init__(self, layout: "cb.Layout", slot_expert, T: int, K: int, H: int, F: int, *, eps: float = 1e-5, p: float = 0.0,
                 gate: str = "softmax", device: Optional[torch.device] = None):
        if gate not in ("softmax", "sigmoid"):
            raise ValueError(gate)
        self.step = RouteStep(layout, T, K, H, device=device, alias_expert_out=False)
        self.T, self.K, self.H, self.F, self.E, self.P = T, K, H, F, layout.E, T * K
        self.eps, self.p = eps, p
        self.gate_flags = cb.GATE_SIGMOID if gate == "sigmoid" else 0
        dev = self.step.device
        self.slot_expert = torch.tensor([int(e) for e in slot_expert], dtype=torch.int32, device=dev)
        if self.slot_expert.numel() != layout.D:
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer (slot_expert size)")

        def new(*shape, dtype=torch.bfloat16):
            return torch.zeros(shape, dtype=dtype, device=dev)

        f32 = torch.float32
        self.gamma, self.beta = torch.ones(H, device=dev), new(H, dtype=f32)
        self.w_router, self.w_gate_up, self.w_down = new(self.E, H), new(self.E, 2 * F, H), new(self.E, H, F)
        self.mean, self.rstd = new(T, dtype=f32), new(T, dtype=f32)
        self.logits = new(T, self.E)
        self.act, self.pre, self.out = new(self.P, F), new(self.P, 2 * F), new(T, H)
        self.grad_pre = new(self.P, 2 * F)              # not `pre` itself: backward may be called again
        self.grad_y, self.grad_expert_out, self.grad_send = new(T, H), new(self.P, H), new(self.P, H)
        self.grad_gate_w, self.grad_logits, self.grad_n, self.grad_x = new(T, K, dtype=f32), new(T, self.E), new(T, H), new(T, H)
        self.grad_gamma, self.grad_beta = new(H, dtype=f32), new(H, dtype=f32)
        self.grad_w_router = new(self.E, H)
        self.grad_w_gate_up, self.grad_w_down = torch.zeros_like(self.w_gate_up), torch.zeros_like(self.w_down)
        ws = max(cb.expert_ffn_workspace_bytes(self.P, layout.D, self.E, H, F), cb.layer_norm_workspace_bytes(T, H), 256)
        self.workspace = torch.empty((ws,), dtype=torch.uint8, device=dev)
        self.x = None                                   # input of the last forward call

    def _experts(self, send: torch.Tensor, expert_out: torch.Tensor) -> None:
        cb.expert_ffn(send, self.step.dest_offsets, self.slot_expert, self.w_gate_up, self.w_down, self.act, expert_out,
                      self.workspace, pre=self.pre)

    def forward(self, x: torch.Tensor, seed: int) -> torch.Tensor:
        """The layer's output for x bfloat16 [T, H] (a buffer of this object, overwritten by the next call).  step.src_rank
        holds the tokens' source ranks; `seed` draws the replica picks and the dropout mask.  x is kept by reference and
        read again by backward; it may be the output buffer itself if no backward call follows."""
        s = self.step
        self.x, self.seed = x, seed
        cb.layer_norm(x, self.gamma, self.beta, self.eps, s.x, self.mean, self.rstd)
        torch.mm(s.x, self.w_router.t(), out=self.logits)
        cb.gate_topk(self.logits, s.topk_ids, s.gate_w, flags=self.gate_flags)
        s.route_fused(seed, experts=self._experts)
        cb.dropout_add(s.y, x, self.p, seed, self.out)
        return self.out

    def backward(self, grad_out: torch.Tensor) -> torch.Tensor:
        """Gradient of x for the last forward call (a buffer of this object); the parameters' gradients are in the grad_*
        attributes.  May be called again for the same forward call, also with a gradient that it returned before."""
        if self.x is None or (self.T > 0 and self.x.data_ptr() == self.out.data_ptr()):
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.backward (no forward call, or its output was written over its input)")
        s = self.step
        cb.dropout_add_backward(grad_out, self.p, self.seed, self.grad_y)
        cb.combine_backward(self.grad_y, s.expert_out, s.row_of_pair, s.gate_w, self.grad_expert_out, self.grad_gate_w)
        cb.expert_ffn_backward(self.grad_expert_out, s.send, s.dest_offsets, self.slot_expert, self.w_gate_up, self.w_down,
                               self.pre, self.act, self.grad_pre, self.workspace, grad_rows=self.grad_send,
                               grad_w_gate_up=self.grad_w_gate_up, grad_w_down=self.grad_w_down)
        cb.permute_backward(self.grad_send, s.row_of_pair, self.K, self.grad_n)
        cb.gate_topk_backward(self.grad_gate_w, self.logits, s.topk_ids, s.gate_w, self.grad_logits, flags=self.gate_flags)
        torch.mm(self.grad_logits.t(), s.x, out=self.grad_w_router)
        torch.addmm(self.grad_n, self.grad_logits, self.w_router, out=self.grad_n)
        cb.layer_norm_backward(self.grad_n, self.x, self.gamma, self.mean, self.rstd, self.grad_n, self.grad_gamma,
                               self.grad_beta, self.workspace)
        # the residual branch; element by element, so grad_out may be grad_x
        return torch.add(self.grad_n, grad_out, out=self.grad_x)
