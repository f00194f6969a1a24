"""One mixture-of-experts layer around the routing step, forward and backward.

    n = norm(x)   logits = n Wr^T   ids, w = gate(logits)   send = route(n, ids)   o = experts(send)
    y = combine(o, w)   out = x + dropout(y)

and, where asked for, a dense block that every token passes beside the experts, whose result joins the residual stream:

    b = x + act(n Wu^T + bu) Wd^T + bd   out = b + dropout(y)

Plumbing only, as in `router`: torch allocates the buffers once, multiplies by the router's weights (a plain library product,
unless router="linear") and adds gradients; everything else is one C-ABI call each, enqueued on the current torch stream.

What a layer needs for its backward pass is 2 T H + 4 P H + 6 P F bytes and more.  `save()` leaves T H bytes of it (the layer's
input rows in 8 bits) and the small arrays of the routing; `restore()` computes the rest again, so that layers of the same sizes
and options may share one object's buffers.  The parameters are attributes that the calls read when they are made, and none is
part of a checkpoint: before each layer's forward and restore calls the user assigns that layer's tensors (gamma, beta, w_*, b_*;
pack_shared() for the 8-bit block), and after its backward call takes the gradients out of grad_* (the next backward call
overwrites them).
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import binding as cb
from .router import RouteStep


@dataclass
class LayerCheckpoint:
    """What `MoELayer.restore` starts from: the layer's input rows in 8 bits (with the residual added, if there was one) and the
    routing's small arrays.  Not the parameters: those of the layer have to be in the object again."""

    rows: Tuple[torch.Tensor, torch.Tensor]        # int8 [T, H], float32 [T, ceil(H / 128)]
    logits: torch.Tensor
    topk_ids: torch.Tensor
    gate_w: torch.Tensor
    src_rank: torch.Tensor
    seed: int


class MoELayer:
    """Parameters, their gradients and the buffers of one layer for T tokens of width H over the experts of `layout`.

    slot_expert: expert of every slot (-1 = empty), as given to the layout.  gate: "softmax" or "sigmoid".
    norm: "layer" (gamma and beta) or "rms" (gamma alone; forward then takes a residual to add first).
    router: "plain" (bfloat16 logits by a library product) or "linear" (float32 logits, with a bias; E a multiple of 8).
    shared: width of the dense block beside the experts, 0 for none; shared_act its activation; shared_8bit runs it with e4m3
    rows and weights (inference only; pack_shared() after the weights have been set).
    Parameters: gamma, beta float32 [H]; w_router bfloat16 [E, H], b_router [E]; w_gate_up [E, 2F, H]; w_down [E, H, F];
    w_shared_up [shared, H], b_shared_up [shared], w_shared_down [H, shared], b_shared_down [H].
    """

    def __init__(self, layout: "cb.Layout", slot_expert, T: int, K: int, H: int, F: int, *, eps: float = 1e-5, p: float = 0.0,
                 gate: str = "softmax", norm: str = "layer", router: str = "plain", shared: int = 0, shared_act: str = "silu",
                 shared_8bit: bool = False, device: Optional[torch.device] = None):
        if gate not in ("softmax", "sigmoid"):
            raise ValueError(gate)
        if norm not in ("layer", "rms"):
            raise ValueError(norm)
        if router not in ("plain", "linear"):
            raise ValueError(router)
        if shared < 0 or shared % 8 != 0 or (shared_8bit and (shared == 0 or shared % 16 != 0 or H % 16 != 0)):
            raise ValueError(f"shared = {shared}")
        if router == "linear" and layout.E % 8 != 0:
            raise ValueError(f"router linear with {layout.E} experts")
        if shared_act not in cb.ACTIVATIONS:
            raise ValueError(shared_act)
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
        self.norm, self.router, self.shared, self.shared_act, self.shared_8bit = norm, router, shared, shared_act, shared_8bit
        self.logits = new(T, self.E, dtype=f32 if router == "linear" else torch.bfloat16)
        self.act, self.pre, self.out = new(self.P, F), new(self.P, 2 * F), new(T, H)
        self.grad_pre = new(self.P, 2 * F)              # not `pre` itself: backward may be called again
        self.grad_y, self.grad_expert_out, self.grad_send = new(T, H), new(self.P, H), new(self.P, H)
        self.grad_gate_w, self.grad_logits, self.grad_n, self.grad_x = new(T, K, dtype=f32), torch.zeros_like(self.logits), new(T, H), new(T, H)
        self.grad_gamma, self.grad_beta = new(H, dtype=f32), new(H, dtype=f32)
        self.grad_w_router = new(self.E, H)
        self.grad_w_gate_up, self.grad_w_down = torch.zeros_like(self.w_gate_up), torch.zeros_like(self.w_down)
        ws = max(cb.expert_ffn_workspace_bytes(self.P, layout.D, self.E, H, F), cb.layer_norm_workspace_bytes(T, H), 256)
        if norm == "rms":
            self.sum = new(T, H)                        # x + residual
            ws = max(ws, cb.rms_norm_workspace_bytes(T, H))
        if router == "linear":
            self.b_router, self.grad_b_router, self.grad_logits16 = new(self.E), new(self.E), new(T, self.E)
            ws = max(ws, cb.linear_workspace_bytes(T, H, self.E))
        if shared > 0:
            self.w_shared_up, self.b_shared_up = new(shared, H), new(shared)
            self.w_shared_down, self.b_shared_down = new(H, shared), new(H)
            self.shared_hidden, self.base = new(T, shared), new(T, H)
            ws = max(ws, cb.linear_workspace_bytes(T, H, shared), cb.linear_workspace_bytes(T, shared, H))
            if shared_8bit:
                def packed(rows, columns):              # e4m3 with one scale a row
                    return new(rows, columns, dtype=torch.float8_e4m3fn), new(rows, 1, dtype=f32)
                self.n8, self.shared_hidden8 = packed(T, H), packed(T, shared)
                self.w_shared_up8, self.w_shared_down8 = packed(shared, H), packed(H, shared)
            else:
                # the block's pre-activation stays in 8 bits up to the backward pass (relu's slope needs its sign, which small values
                # lose there)
                self.shared_pre = new(T, shared) if shared_act == "relu" else (new(T, shared, dtype=torch.int8),
                                                                               new(T, -(-shared // cb.PACK_GROUP), dtype=f32))
                self.grad_shared = new(T, shared)
                self.grad_w_shared_up, self.grad_b_shared_up = torch.zeros_like(self.w_shared_up), new(shared)
                self.grad_w_shared_down, self.grad_b_shared_down = torch.zeros_like(self.w_shared_down), new(H)
        if router == "linear" or shared > 0:
            self.grad_n_dense = new(T, H)
        self.workspace = torch.empty((ws,), dtype=torch.uint8, device=dev)
        self.x = None                                   # input of the last forward call
        self.x_restored = None                          # restored rows, allocated by the first restore()

    def _experts(self, send: torch.Tensor, expert_out: torch.Tensor) -> None:
        cb.expert_ffn(send, self.step.dest_offsets, self.slot_expert, self.w_gate_up, self.w_down, self.act, expert_out,
                      self.workspace, pre=self.pre)

    def pack_shared(self) -> None:
        """The dense block's weights in 8 bits (shared_8bit), from w_shared_up and w_shared_down as they are now."""
        cb.pack_rows(self.w_shared_up, *self.w_shared_up8)
        cb.pack_rows(self.w_shared_down, *self.w_shared_down8)

    def _norm(self, x: torch.Tensor, residual: Optional[torch.Tensor]) -> torch.Tensor:
        """Fills step.x (and n8); returns the rows that were normalised."""
        s = self.step
        packed = self.n8 if self.shared_8bit else None
        if self.norm == "layer":
            if residual is not None:
                raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.forward (a residual needs norm=\"rms\")")
            cb.layer_norm(x, self.gamma, self.beta, self.eps, s.x, self.mean, self.rstd)
            if packed is not None:
                cb.pack_rows(s.x, *packed)
            return x
        cb.rms_norm(x, self.gamma, self.eps, residual=residual, sum_out=None if residual is None else self.sum, y=s.x, packed=packed,
                    rstd=self.rstd)
        return x if residual is None else self.sum

    def _shared_up(self) -> None:
        if self.shared_8bit:
            cb.linear(self.n8, self.w_shared_up8, self.shared_hidden, self.workspace, bias=self.b_shared_up, act=self.shared_act)
            cb.pack_rows(self.shared_hidden, *self.shared_hidden8)
        else:
            cb.linear(self.step.x, self.w_shared_up, self.shared_hidden, self.workspace, bias=self.b_shared_up, act=self.shared_act,
                      pre=self.shared_pre)

    def forward(self, x: torch.Tensor, seed: int, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The layer's output for x bfloat16 [T, H] (a buffer of this object, overwritten by the next call).  step.src_rank
        holds the tokens' source ranks; `seed` draws the replica picks and the dropout mask.  residual (norm "rms") is added to x
        first: the layer's input is their sum, x alone is not kept.  Otherwise x is kept by reference and read again by
        backward; it may be the output buffer itself if no backward call follows."""
        s = self.step
        self.x, self.seed = self._norm(x, residual), seed
        x = self.x
        if self.router == "plain":
            torch.mm(s.x, self.w_router.t(), out=self.logits)
        else:
            cb.linear(s.x, self.w_router, self.logits, self.workspace, bias=self.b_router)
        cb.gate_topk(self.logits, s.topk_ids, s.gate_w, flags=self.gate_flags)
        s.route_fused(seed, experts=self._experts)
        if self.shared > 0:
            self._shared_up()
            hidden, w = (self.shared_hidden8, self.w_shared_down8) if self.shared_8bit else (self.shared_hidden, self.w_shared_down)
            cb.linear(hidden, w, self.base, self.workspace, bias=self.b_shared_down, residual=x)
            x = self.base
        cb.dropout_add(s.y, x, self.p, seed, self.out)
        return self.out

    def save(self) -> LayerCheckpoint:
        """What restore() needs of the last forward call, in buffers of its own."""
        if self.x is None or (self.T > 0 and self.x.data_ptr() == self.out.data_ptr()):
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.save (no forward call, or its output was written over its input)")
        s, dev = self.step, self.step.device
        rows = (torch.empty((self.T, self.H), dtype=torch.int8, device=dev),
                torch.empty((self.T, -(-self.H // cb.PACK_GROUP)), dtype=torch.float32, device=dev))
        cb.pack_rows(self.x, *rows)
        seed = self.seed.clone() if isinstance(self.seed, torch.Tensor) else self.seed
        return LayerCheckpoint(rows, self.logits.clone(), s.topk_ids.clone(), s.gate_w.clone(), s.src_rank.clone(), seed)

    def restore(self, checkpoint: LayerCheckpoint) -> None:
        """Computes again what backward needs, with the routing as it was and the rows as they were kept, rounded to bfloat16.  backward
        then gives the gradients at those rows; of the checkpoint it reads a seed on the device only.  step.src_rank is the checkpoint's
        afterwards."""
        s, c = self.step, checkpoint
        if tuple(c.rows[0].shape) != (self.T, self.H) or c.logits.shape != self.logits.shape or c.topk_ids.shape != s.topk_ids.shape:
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.restore (sizes)")
        if self.x_restored is None:
            self.x_restored = torch.empty((self.T, self.H), dtype=torch.bfloat16, device=s.device)
        cb.unpack_rows(*c.rows, self.x_restored)
        self.x, self.seed = self._norm(self.x_restored, None), c.seed
        self.logits.copy_(c.logits)
        s.topk_ids.copy_(c.topk_ids)
        s.gate_w.copy_(c.gate_w)
        s.src_rank.copy_(c.src_rank)
        s.route_fused(c.seed, experts=self._experts)
        if self.shared > 0:
            self._shared_up()

    def backward(self, grad_out: torch.Tensor) -> torch.Tensor:
        """Gradient of x (and of residual) for the last forward or restore call (a buffer of this object); the parameters' gradients
        are in the grad_* attributes.  May be called again for the same forward call, also with a gradient that it returned before."""
        if self.x is None or (self.T > 0 and self.x.data_ptr() == self.out.data_ptr()):
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.backward (no forward call, or its output was written over its input)")
        if self.shared_8bit:
            raise cb.CobaltError(cb.ERR_INVALID_ARG, "MoELayer.backward (shared_8bit is for inference)")
        s = self.step
        cb.dropout_add_backward(grad_out, self.p, self.seed, self.grad_y)
        cb.combine_backward(self.grad_y, s.expert_out, s.row_of_pair, s.gate_w, self.grad_expert_out, self.grad_gate_w)
        cb.expert_ffn_backward(self.grad_expert_out, s.send, s.dest_offsets, self.slot_expert, self.w_gate_up, self.w_down,
                               self.pre, self.act, self.grad_pre, self.workspace, grad_rows=self.grad_send,
                               grad_w_gate_up=self.grad_w_gate_up, grad_w_down=self.grad_w_down)
        cb.permute_backward(self.grad_send, s.row_of_pair, self.K, self.grad_n)
        cb.gate_topk_backward(self.grad_gate_w, self.logits, s.topk_ids, s.gate_w, self.grad_logits, flags=self.gate_flags)
        if self.router == "plain":
            torch.mm(self.grad_logits.t(), s.x, out=self.grad_w_router)
            torch.addmm(self.grad_n, self.grad_logits, self.w_router, out=self.grad_n)
        else:
            cb.linear_backward(self.grad_logits, s.x, self.w_router, self.workspace, grad_pre=self.grad_logits16, grad_x=self.grad_n_dense,
                               grad_w=self.grad_w_router, grad_bias=self.grad_b_router)
            self.grad_n.add_(self.grad_n_dense)
        if self.shared > 0:
            cb.linear_backward(grad_out, self.shared_hidden, self.w_shared_down, self.workspace, grad_x=self.grad_shared,
                               grad_w=self.grad_w_shared_down, grad_bias=self.grad_b_shared_down)
            cb.linear_backward(self.grad_shared, s.x, self.w_shared_up, self.workspace, act=self.shared_act, pre=self.shared_pre,
                               grad_pre=self.grad_shared, grad_x=self.grad_n_dense, grad_w=self.grad_w_shared_up,
                               grad_bias=self.grad_b_shared_up)
            self.grad_n.add_(self.grad_n_dense)
        if self.norm == "rms":                          # the gradient down the residual stream joins in the same pass
            cb.rms_norm_backward(self.grad_n, self.x, self.gamma, self.rstd, self.grad_x, self.grad_gamma, self.workspace, grad_sum=grad_out)
            return self.grad_x
        cb.layer_norm_backward(self.grad_n, self.x, self.gamma, self.mean, self.rstd, self.grad_n, self.grad_gamma,
                               self.grad_beta, self.workspace)
        # the residual branch; element by element, so grad_out may be grad_x
        return torch.add(self.grad_n, grad_out, out=self.grad_x)
