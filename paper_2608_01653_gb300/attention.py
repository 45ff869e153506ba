"""An attention layer whose weights and cache are 4-bit: the operators of hatq run together as a model uses them, for
prompts, pieces of prompts and single tokens.

  c, s    = quantize_tokens(x, hb)                       INT8 codes of the tokens, one scale each
  q, k, v = linear4(c, qkv, scales=s)                    columns of one buffer
  q, k    = turn(q, k)                                   positions, if the model has any (the caller's)
  append_tokens(cache, k, v, table, lengths, starts)
  y       = attend_tokens(q, cache, table, lengths, starts)
  c, s    = quantize_tokens(y, hb)
  out     = linear4(c, o, scales=s)

No arithmetic happens here. Everything is enqueued on the current stream without a look at the device's values, so a
step can be captured in a CUDA graph; shapes depend on the number of rows only.
"""
from __future__ import annotations

from . import hatq


class AttentionBlock:
    """heads query heads over kv_heads key and value heads of `width`, C values a token.

    w_qkv [(heads + 2 kv_heads) * width][C] (queries first, then keys, then values) and w_o [C][heads * width], floating
    point; both are transformed along their inputs in blocks of hb (a power of two that divides C and heads * width) and
    quantized to 4 bits with a scale per channel and `group` inputs."""

    def __init__(self, w_qkv, w_o, heads, kv_heads, width, hb, group=128):
        n, c = w_qkv.shape
        if kv_heads < 1 or heads % kv_heads or n != (heads + 2 * kv_heads) * width:
            raise ValueError(f"w_qkv: {n} rows for {heads} + 2 x {kv_heads} heads of {width}")
        if tuple(w_o.shape) != (c, heads * width):
            raise ValueError(f"w_o: shape {tuple(w_o.shape)}, expected {(c, heads * width)}")
        self.heads, self.kv_heads, self.width, self.hb = heads, kv_heads, width, hb
        self.qkv = hatq.prepare_linear4(w_qkv, group=group, hb=hb)
        self.o = hatq.prepare_linear4(w_o, group=group, hb=hb)

    def cache(self, pages, page=64, device="cuda"):
        """An empty cache of this layer's sizes."""
        return hatq.TokenCache.empty(pages, self.kv_heads, self.width, page=page, device=device)

    def forward(self, x, cache, table, lengths, starts=None, turn=None):
        """x [rows][C] in float16 or bfloat16, the newest tokens of every sequence (table, lengths, starts as hatq.append_tokens
        takes them; they go into the cache). turn(q, k), if given, returns both with their positions (k as it was given).
        Returns [rows][C] in x's type; what it holds for rows of no sequence (padding behind the last) means nothing."""
        torch = hatq._token_torch()
        types = torch.float16, torch.bfloat16
        if x.dtype not in types:                                            # (append would take it, attention would not)
            raise ValueError(f"x: dtype {x.dtype}, expected float16 or bfloat16")
        rows, h, kv, d = x.shape[0], self.heads, self.kv_heads, self.width
        c, s = hatq.quantize_tokens(x, hb=self.hb, codes="f16")
        y = hatq.linear4(c, self.qkv, scales=s, dtype=x.dtype).view(rows, h + 2 * kv, d)
        q, k, v = y[:, :h], y[:, h:h + kv], y[:, h + kv:]
        if turn is not None:
            q, k = turn(q, k)
            if q.dtype not in types or tuple(q.shape) != (rows, h, d) or q.device != x.device or q.stride(2) != 1:
                raise ValueError(f"turn: q is {q.dtype} {tuple(q.shape)} on {q.device} with strides {q.stride()}, expected float16 or "
                                 f"bfloat16 {(rows, h, d)} on {x.device} with contiguous heads")
        hatq.append_tokens(cache, k, v, table, lengths, starts)
        y = hatq.attend_tokens(q, cache, table, lengths, starts)
        c, s = hatq.quantize_tokens(y.reshape(rows, h * d), hb=self.hb, codes="f16")
        return hatq.linear4(c, self.o, scales=s, dtype=x.dtype)
