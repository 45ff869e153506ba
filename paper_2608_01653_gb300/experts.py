"""A feed-forward block of experts in 8-bit integers: the token operators run
together as a model uses them, for prompts and for single tokens.

Tokens are sent to experts (`plan`), copied in expert order while they are
transformed and quantized (one scale per token), multiplied by the experts' gate
and up matrices, activated and gated while they are quantized again, multiplied
by the down matrices, and added up per token with the router's weights:

  rows, offsets, slots = plan(ids, experts)
  q, s  = quantize_tokens(x, hb, rows=rows)
  h     = grouped_linear(q, s, offsets, gate_up)         [rows][2 F]
  q, s  = quantize_tokens(h, hb, act="silu", gated=True)
  z     = grouped_linear(q, s, offsets, down)            [rows][C]
  y     = combine_rows(z, slots, weights)                [tokens][C]

No arithmetic happens here. Everything is enqueued on the current stream
without a look at the device's values, so a step can be captured in a CUDA
graph; shapes depend on the number of tokens only.
"""
from __future__ import annotations

from . import hatq


def plan(ids, experts):
    """Where each (token, choice) goes: ids is an integer tensor [tokens][topk]; an id outside [0, experts) is a choice
    that no expert takes. Returns int32 tensors: rows [tokens * topk], the token of each row in expert order (choices
    that no expert takes come last), offsets [experts + 1], and slots [tokens][topk], the row of each choice (-1: none)."""
    import torch
    flat = ids.reshape(-1).long()
    taken = (flat >= 0) & (flat < experts)
    key = torch.where(taken, flat, experts)
    order = torch.argsort(key, stable=True)
    ends = torch.searchsorted(key[order], torch.arange(experts + 1, device=ids.device), right=False)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(order.numel(), device=ids.device)
    slots = torch.where(taken, slots, -1).reshape(ids.shape)
    return (order // ids.shape[-1]).to(torch.int32), ends.to(torch.int32), slots.to(torch.int32)


class ExpertBlock:
    """experts feed-forward layers C -> F -> C with a gated activation.

    w_gate_up [experts][2 F][C] (gate rows first), w_down [experts][C][F], floating point; they are transformed along
    their inputs in blocks of hb_in / hb_mid (powers of two that divide C / F) and quantized per output channel."""

    def __init__(self, w_gate_up, w_down, hb_in, hb_mid, act="silu"):
        e, f2, c = w_gate_up.shape
        if w_down.shape != (e, c, f2 // 2) or f2 % 2:
            raise ValueError(f"w_down: shape {tuple(w_down.shape)}, expected {(e, c, f2 // 2)}")
        self.experts, self.hb_in, self.hb_mid, self.act = e, hb_in, hb_mid, act
        self.gate_up = hatq.prepare_linear(w_gate_up, hb=hb_in)
        self.down = hatq.prepare_linear(w_down, hb=hb_mid)

    def forward(self, x, ids, weights):
        """x [tokens][C]; ids and float32 weights [tokens][topk] from the router. Returns [tokens][C] in x's type."""
        rows, offsets, slots = plan(ids, self.experts)
        q, s = hatq.quantize_tokens(x, hb=self.hb_in, rows=rows, codes="f16")
        h = hatq.grouped_linear(q, s, offsets, self.gate_up, dtype=x.dtype)
        q, s = hatq.quantize_tokens(h, hb=self.hb_mid, act=self.act, gated=True, codes="f16")
        z = hatq.grouped_linear(q, s, offsets, self.down, dtype=x.dtype)
        return hatq.combine_rows(z, slots, weights)
