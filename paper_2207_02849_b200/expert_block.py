"""A residual block with experts, trained: the norms with gate and residual scale, the experts' products and the 8-bit
checkpoint of their hidden layer, as one differentiable step.

    u = N(x) w + ...;  z = up_e u;  a = act(z)  (or act(z_gate) z_value);  y = down_e a;  x' = x + s a(g) N(y) w';  u' = N(x') w''

for rows sorted by expert.  Of blocks in a row, each makes the next one's u with its own exit norm.  Between forward and backward
a block keeps x, x', u, y and the checkpoint (q, scales) of z (x only where it made its u itself); the hidden activation is made
again from the checkpoint.  Gradients are what the finite-difference approximation of a
best-response Jacobian needs: two gradients at displaced parameters (arXiv 2207.02849, Sec. 3.2)."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as bt


class ExpertBlock:
    """Shapes, descriptors and workspace of a block of `n_experts` experts of hidden width `hidden` on rows of width `d`.

    Parameters are the caller's: a dict with `entry` [3 or 5, d] and `exit` [3 or 5, d] fp32 (see BlockNorm; the entry
    uses w_pre of `entry`, the exit w_post, the residual scale and, for the next block's norm, w_pre of `exit`),
    `up` [n_experts, hidden or 2 * hidden, d] and `down` [n_experts, d, hidden] in the operand type."""

    def __init__(self, n_experts: int, d: int, hidden: int, rows: int, dtype: torch.dtype = torch.bfloat16, act: int = bt.ACT_SILU,
                 gated: bool = True, norm: int = bt.NORM_RMS, gate: int = bt.GATE_NONE, rows_per_gate: int = 1, eps: float = 1e-6,
                 bias: bool = False, device="cuda"):
        code = {torch.bfloat16: bt.BETTY_BF16, torch.float16: bt.BETTY_F16}.get(dtype)
        if code is None:
            raise ValueError(f"an expert block's operands are bf16 or fp16, got {dtype}")
        self.d, self.hidden, self.rows, self.dtype, self.device = int(d), int(hidden), int(rows), dtype, device
        self.act8 = bt.Act8(hidden, act=act, gated=gated)
        self.entry = bt.BlockNorm(d, pre=norm, post=bt.NORM_NONE, eps=eps, bias=bias)
        self.exit = bt.BlockNorm(d, pre=norm, post=norm, gate=gate, rows_per_gate=rows_per_gate, eps=eps, bias=bias)
        self.up = bt.Grouped(n_experts, d, self.act8.width, code)
        self.down = bt.Grouped(n_experts, hidden, d, code)
        # the block's own matrices are contiguous: only x, its gradient and the gate can be the caller's slices
        need = max(bt.betty_block_norm_workspace_size(self.entry, rows, False), bt.betty_block_norm_workspace_size(self.exit, rows, False),
                   bt.betty_grouped_workspace_size(self.up, rows), bt.betty_grouped_workspace_size(self.down, rows))
        self.ws = bt.Workspace.of_bytes(need, device)

    def _rows(self, width: int, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
        return torch.empty(self.rows, width, dtype=dtype or self.dtype, device=self.device)

    def forward(self, p: dict, offsets: torch.Tensor, x: torch.Tensor, gate: Optional[torch.Tensor] = None,
                u: Optional[torch.Tensor] = None, next_norm: bool = True):
        """(x', u', kept): the residual stream, the next block's normed input and what `backward` needs.  `u`: the normed input
        that the block before has made (its u', with its `exit` w_pre); None: it is made here, with `entry`.  next_norm False:
        no block follows, u' is None."""
        z, a, y = self._rows(self.act8.width), self._rows(self.hidden), self._rows(self.d)
        q, scales = self.act8.empty(self.rows, self.device)
        x_out, u_out, own_norm = torch.empty_like(x), self._rows(self.d) if next_norm else None, u is None
        if own_norm:
            u = self._rows(self.d)
            bt.betty_block_norm(self.entry, p["entry"], x, None, None, None, u)
        bt.betty_grouped_forward(self.up, offsets, u, p["up"], z, self.ws)
        bt.betty_act8_store(self.act8, z, a, q, scales)
        bt.betty_grouped_forward(self.down, offsets, a, p["down"], y, self.ws)
        bt.betty_block_norm(self.exit, p["exit"], x, y, gate, x_out, u_out)
        return x_out, u_out, {"x": x if own_norm else None, "x_out": x_out, "u": u, "y": y, "q": q, "scales": scales, "gate": gate}

    def backward(self, p: dict, offsets: torch.Tensor, kept: dict, dx_out: Optional[torch.Tensor], du_out: Optional[torch.Tensor],
                 weight_dtype: torch.dtype = torch.float32) -> dict:
        """Gradients of x, gate and the parameters from those of x' and u' (either may be None).  Where `forward` was given u: its
        gradient under "u", "x" without what goes through u, and no "entry": the block before takes them as du_out and dx_out."""
        x, gate = kept["x"], kept["gate"]
        dx, dy, da, dz, a, du = (torch.empty_like(kept["x_out"]), self._rows(self.d), self._rows(self.hidden), self._rows(self.act8.width),
                                 self._rows(self.hidden), self._rows(self.d))
        grads = {"exit": torch.empty_like(p["exit"]),
                 "up": torch.empty(p["up"].shape, dtype=weight_dtype, device=self.device),
                 "down": torch.empty(p["down"].shape, dtype=weight_dtype, device=self.device),
                 "gate": torch.empty_like(gate) if gate is not None else None, "x": dx}
        bt.betty_block_norm_backward(self.exit, p["exit"], kept["x_out"], kept["y"], gate, du_out, dx_out, dx, dy, grads["gate"],
                                     grads["exit"], self.ws)
        bt.betty_grouped_backward_data(self.down, offsets, dy, p["down"], da, self.ws)
        bt.betty_act8_backward(self.act8, kept["q"], kept["scales"], da, dz, a)
        bt.betty_grouped_backward_weight(self.down, offsets, dy, a, grads["down"], self.ws)
        bt.betty_grouped_backward_weight(self.up, offsets, dz, kept["u"], grads["up"], self.ws)
        bt.betty_grouped_backward_data(self.up, offsets, dz, p["up"], du, self.ws)
        if x is None:
            grads["u"] = du
        else:
            grads["entry"] = torch.empty_like(p["entry"])
            bt.betty_block_norm_backward(self.entry, p["entry"], x, None, None, du, dx, dx, None, None, grads["entry"], self.ws)
        return grads
