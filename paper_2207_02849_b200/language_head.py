"""The head of a language model with its losses, trained: logits W u over a vocabulary, which are not kept, and one loss per row.

    z = W u / T;   cross entropy with target tokens, or the divergence from a teacher's top logits;   loss[rows]

u is what the last block hands on (ExpertBlock's u').  A cost is a weighted sum of the row losses: `backward` takes the weights, and
the row losses are the cost's gradient by them, which is what a problem above that weighs the rows needs for its best-response
Jacobian by finite differences (arXiv 2207.02849, Sec. 3.2): two forward passes at displaced parameters."""
from __future__ import annotations

import torch

from . import binding as bt


class LanguageHead:
    """Descriptors and workspace of a head of `vocab` tokens on up to `rows` rows of width `d`.

    W [vocab, d] is the caller's, in the operand type.  any_layout: W may be a slice of a wider or longer buffer, whose rows do not start
    on 16-byte boundaries; the workspace has room for its aligned copy (vocab * d values) then.  Without it such a W is refused (of a
    d that is not a multiple of 8 the copy is needed in any case).  `top`: entries a row that a teacher brings at most (0: no teacher);
    `temperature` divides both the teacher's and the head's logits of the distillation; smoothing and z_loss belong to
    the cross entropy (see VocabLoss)."""

    def __init__(self, vocab: int, d: int, rows: int, top: int = 0, dtype: torch.dtype = torch.bfloat16, temperature: float = 1.0,
                 smoothing: float = 0.0, z_loss: float = 0.0, device="cuda", any_layout: bool = True):
        code = {torch.bfloat16: bt.BETTY_BF16, torch.float16: bt.BETTY_F16}.get(dtype)
        if code is None:
            raise ValueError(f"a language head's operands are bf16 or fp16, got {dtype}")
        self.vocab, self.d, self.rows, self.top, self.dtype, self.device = int(vocab), int(d), int(rows), int(top), dtype, device
        self.tokens = bt.VocabLoss(vocab, d, code, smoothing=smoothing, z_loss=z_loss)
        self.teacher = bt.VocabLoss(vocab, d, code, temperature=temperature)
        self.any_layout = bool(any_layout) or self.d % 8 != 0
        self.ws = bt.Workspace.of_bytes(max(bt.betty_vocab_workspace_size(self.tokens, rows, 0, self.any_layout),
                                            bt.betty_vocab_workspace_size(self.teacher, rows, top, self.any_layout)), device)

    def _check_layout(self, w: torch.Tensor) -> None:
        """Forward and backward take the same W: what only some calls would find room for is refused by all."""
        if not self.any_layout and (w.data_ptr() % 16 != 0 or (self.vocab > 1 and w.stride(0) % 8 != 0)):
            raise ValueError("the rows of w do not start on 16-byte boundaries, and the head was made without room for an aligned copy (any_layout)")

    def _losses(self, u: torch.Tensor):
        return torch.empty(2, u.shape[0], dtype=torch.float32, device=u.device).unbind(0)

    def forward(self, w: torch.Tensor, u: torch.Tensor, target: torch.Tensor):
        """(loss [rows], kept) against the tokens `target` (int32 or int64; outside the vocabulary: the row is left out)."""
        self._check_layout(w)
        loss, lse = self._losses(u)
        bt.betty_vocab_ce(self.tokens, u, w, target, loss, lse, self.ws)
        return loss, {"u": u, "lse": lse, "target": target}

    def forward_teacher(self, w: torch.Tensor, u: torch.Tensor, ids: torch.Tensor, logits: torch.Tensor):
        """(loss [rows], kept) against a teacher's top logits (ids, logits) [rows, entries]; an id outside the vocabulary is no entry."""
        if ids.dim() == 2 and ids.shape[1] > self.top:
            raise ValueError(f"the head was made for {self.top} entries a row, got {ids.shape[1]}")
        self._check_layout(w)
        loss, lse = self._losses(u)
        bt.betty_vocab_distill(self.teacher, u, w, ids, logits, loss, lse, self.ws)
        return loss, {"u": u, "lse": lse, "ids": ids, "logits": logits}

    def backward(self, w: torch.Tensor, kept: dict, dloss: torch.Tensor, wants=("u", "w"), weight_dtype: torch.dtype = torch.float32) -> dict:
        """Gradients of sum(dloss * loss) by u and w, those of `wants`."""
        self._check_layout(w)
        u = kept["u"]
        du = torch.empty(u.shape, dtype=u.dtype, device=u.device) if "u" in wants else None
        dw = torch.empty(w.shape, dtype=weight_dtype, device=w.device) if "w" in wants else None
        if "ids" in kept:
            bt.betty_vocab_distill_backward(self.teacher, u, w, kept["ids"], kept["logits"], kept["lse"], dloss, du, dw, self.ws)
        else:
            bt.betty_vocab_ce_backward(self.tokens, u, w, kept["target"], kept["lse"], dloss, du, dw, self.ws)
        return {k: v for k, v in (("u", du), ("w", dw)) if v is not None}
