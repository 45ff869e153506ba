"""Token operators at their edges: empty sources, ragged ends, every tile of the product kernel, several host threads.

References in 64 bits; bounds as derived in check_quantized of test_gpu_tokens.py.
"""
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H
from tests.test_gpu_tokens import CODES, TYPES, check_quantized, finish, gen

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ quantize_tokens

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("rows,c,hb", [(1500, 2000, 16), (1500, 2001, 1), (900, 2048, 64), (200, 16384, 256), (150, 9001, 1)])
def test_quantize_rows_without_a_source(dtype, kind, rows, c, hb):
    """No source row at all: nothing may be read, and every row is an empty one."""
    x = torch.empty(0, c, dtype=TYPES[dtype], device="cuda")
    index = torch.randint(-1, 2, (rows,), generator=gen(1), device="cuda").to(torch.int32)
    q, s = H.quantize_tokens(x, hb=hb, rows=index, codes=kind)
    finish()
    assert q.shape == (rows, c) and bool((q == 0).all()) and bool((s == 1).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("c", [1032, 1992, 2001, 2047, 2056])
def test_quantize_rows_that_end_inside_a_warp(dtype, gated, c):
    """Many rows on 16-byte boundaries whose last values end anywhere in a thread's 32; some rows are empty."""
    rows, width = 1600, c * (1 + gated)
    pitch = -(-width // 8) * 8
    x = torch.randn(rows, pitch, generator=gen(2), device="cuda").to(TYPES[dtype])[:, :width]
    index = torch.randint(-1, rows + 1, (rows,), generator=gen(3), device="cuda").to(torch.int32)
    act = "silu" if gated else "none"
    for at in (None, index):
        q, s = H.quantize_tokens(x, act=act, gated=gated, rows=at, codes="f16")
        finish()
        check_quantized(x, q, s, 1, act, gated, at)
