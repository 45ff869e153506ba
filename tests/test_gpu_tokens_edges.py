"""Token operators at their edges: empty sources, ragged ends, every tile of the product kernel, several host threads.

References in 64 bits; bounds as derived in check_quantized of test_gpu_tokens.py.
"""
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H
from tests.test_gpu_tokens import (CODES, TYPES, check_quantized, codes, finish, gen, grouped_reference, integer_sums,
                                   offsets_of)

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


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("rows,c,hb", [(400, 9000, 8), (333, 12345, 1), (160, 32768, 256), (2000, 1000, 4), (40_000, 40, 8)])
def test_quantize_many_rows_with_an_activation(dtype, act, rows, c, hb):
    """More rows than are at work at a time, on and off 16-byte boundaries, wider and narrower than a warp's values."""
    x = (4 * torch.randn(rows, c, generator=gen(12), device="cuda")).to(TYPES[dtype])
    index = torch.randint(-1, rows + 1, (rows,), generator=gen(13), device="cuda").to(torch.int32)
    for at, kind in ((None, "i8"), (index, "f16")):
        q, s = H.quantize_tokens(x, hb=hb, act=act, rows=at, codes=kind)
        finish()
        check_quantized(x, q, s, hb, act, rows=at)


# ------------------------------------------------------------------ products on pairs of CTAs

def padded(rows, k, seed):
    """fp16 codes whose rows lie on 16-byte boundaries, as the copy engine takes them, whatever k."""
    return torch.zeros(rows, -(-k // 8) * 8, dtype=torch.float16, device="cuda")[:, :k].copy_(codes(rows, k, seed, "f16"))


@pytest.mark.parametrize("rows,k,n", [(1300, 4096, 4224), (2500, 64, 4096), (4001, 2100, 3970)])
def test_products_on_pairs_again_and_again(rows, k, n):
    """Two operands in turn through the same tiles: a half of the tokens read before it has arrived would be the other's."""
    xs = [padded(rows, k, seed) for seed in (4, 5)]
    w, one = codes(n, k, 6), torch.ones(max(rows, n), device="cuda")
    L, s = H.prepare_linear(w, scales=one[:n]), one[:rows].contiguous()
    refs = [integer_sums(x, w).float() for x in xs]
    ys = [H.linear(xs[i % 2], s, L, dtype=torch.float32) for i in range(20)]
    finish()
    assert all(torch.equal(y, refs[i % 2]) for i, y in enumerate(ys))


RAGGED = [1500, 0, 31, 193, 2100, 1, 191, 33, 0, 640, 1000, 700]


def test_grouped_products_on_pairs_again_and_again():
    k, n, e = 1024, 1500, len(RAGGED)
    rows = sum(RAGGED)
    xs = [codes(rows, k, seed, "f16") for seed in (7, 8)]
    w, off, one = codes(e * n, k, 9).view(e, n, k), offsets_of(RAGGED), torch.ones(rows, device="cuda")
    L = H.prepare_linear(w, scales=torch.ones(e, n, device="cuda"))
    refs = [grouped_reference(x, w, off) for x in xs]
    ys = [H.grouped_linear(xs[i % 2], one, off, L, dtype=torch.float32) for i in range(20)]
    finish()
    assert all(torch.equal(y, refs[i % 2]) for i, y in enumerate(ys))


def test_grouped_products_on_pairs_behind_an_expired_wait():
    """Skipped, with every copy that was asked for waited for; right again after the status was read."""
    k, n, e = 512, 1500, len(RAGGED)
    rows = sum(RAGGED)
    x, w, off = codes(rows, k, 10, "f16"), codes(e * n, k, 11).view(e, n, k), offsets_of(RAGGED)
    one, L = torch.ones(rows, device="cuda"), H.prepare_linear(w, scales=torch.ones(e, n, device="cuda"))
    finish()
    out = torch.full((rows, n), 3.0, device="cuda")
    H.selftest_wait(1000)
    H.grouped_linear(x, one, off, L, out=out)
    torch.cuda.synchronize()
    with pytest.raises(H.HatqError) as error:
        H.sync_status()
    assert error.value.status == H.ERR_TIMEOUT and bool((out == 3).all())
    H.grouped_linear(x, one, off, L, out=out)
    finish()
    assert torch.equal(out, grouped_reference(x, w, off))


def test_products_of_every_kind_follow_one_another():
    """Kernels with other tiles and barriers start on the same SMs at once: nothing of the one before may still arrive."""
    calls = []
    for i, (rows, k, n, kind) in enumerate([(2500, 64, 4096, "f16"), (40, 4096, 300, "f16"), (60, 700, 300, "i8"),
                                            (1300, 1024, 4224, "f16"), (2, 512, 100, "i8"), (300, 256, 2100, "f16")]):
        x, w, one = codes(rows, k, 20 + i, kind), codes(n, k, 30 + i), torch.ones(max(rows, n), device="cuda")
        calls.append((x, one[:rows].contiguous(), H.prepare_linear(w, scales=one[:n]), integer_sums(x, w).float()))
    ys = []
    for turn in range(12):
        order = calls[turn % 6:] + calls[:turn % 6]
        ys += [(H.linear(x, s, L, dtype=torch.float32), ref) for x, s, L, ref in (order if turn % 2 else order[::-1])]
    finish()
    assert all(torch.equal(y, ref) for y, ref in ys)


# ------------------------------------------------------------------ products of a few rows

@pytest.mark.parametrize("rows,k,n,kind", [(1, 4096, 4096, "i8"), (2, 300, 77, "f16"), (8, 512, 256, "i8")])
def test_a_few_rows_behind_an_expired_wait(rows, k, n, kind):
    """As with many rows: the output is left alone until the status was read."""
    x, w, one = codes(rows, k, 40, kind), codes(n, k, 41), torch.ones(n, device="cuda")
    L, G, off = H.prepare_linear(w, scales=one), H.prepare_linear(w[None], scales=one[None]), offsets_of([rows])
    s = one[:rows].contiguous()
    finish()
    a, b = torch.full((rows, n), 3.0, device="cuda"), torch.full((rows, n), 3.0, device="cuda")
    H.selftest_wait(1000)
    H.linear(x, s, L, out=a)
    H.grouped_linear(x, s, off, G, out=b)
    torch.cuda.synchronize()
    with pytest.raises(H.HatqError) as error:
        H.sync_status()
    assert error.value.status == H.ERR_TIMEOUT and bool((a == 3).all()) and bool((b == 3).all())
    H.linear(x, s, L, out=a)
    H.grouped_linear(x, s, off, G, out=b)
    finish()
    ref = integer_sums(x, w).float()
    assert torch.equal(a, ref) and torch.equal(b, ref)


# ------------------------------------------------------------------ weights

def test_scales_and_bias_in_another_order_are_refused():
    """[n][experts] holds as many values as [experts][n], in the wrong order."""
    w, one = codes(4 * 6, 32, 60).view(4, 6, 32), torch.ones(4, 6, device="cuda")
    for bad in (one.T, one.T.contiguous(), one.view(2, 12), one.view(3, 8), one[:, None]):
        with pytest.raises(ValueError):
            H.prepare_linear(w, scales=bad)
        with pytest.raises(ValueError):
            H.prepare_linear(w, scales=one, bias=bad)
    with pytest.raises(ValueError):
        H.prepare_linear(w[0], scales=one[0].view(2, 3))
    x, s, off = codes(9, 32, 61), one.new_ones(9), offsets_of([1, 4, 0, 4])
    scales = torch.rand(4, 6, generator=gen(62), device="cuda")
    ys = [H.grouped_linear(x, s, off, H.prepare_linear(w, scales=v), dtype=torch.float32)
          for v in (scales, scales.view(24), scales[:, :, None], scales.double())]
    zs = [H.linear(x, s, H.prepare_linear(w[1], scales=v), dtype=torch.float32) for v in (scales[1], scales[1:2], scales[1][:, None])]
    finish()
    assert all(torch.equal(y, ys[0]) for y in ys) and all(torch.equal(z, zs[0]) for z in zs)
    assert torch.equal(zs[0][1:5], ys[0][1:5])


# ------------------------------------------------------------------ combine_rows

@pytest.mark.parametrize("dtype,c", [("f32", (1 << 29) + 1), ("f16", (1 << 30) + 8), ("bf16", (1 << 30) + 3)])
def test_combine_rows_of_more_than_2_gb(dtype, c):
    """A row whose bytes do not count in 32 bits; one row with weight 1 is the row itself."""
    y = torch.empty(1, c, dtype=TYPES[dtype], device="cuda")
    step = 1 << 27
    for at in range(0, c, step):
        y[0, at:at + step].normal_(generator=gen(at // step))
    out = H.combine_rows(y, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, 1, device="cuda"))
    finish()
    assert torch.equal(out, y)


# ------------------------------------------------------------------ columns of one buffer

@pytest.mark.parametrize("rows", [1, 2, 40, 700])
@pytest.mark.parametrize("left", [False, True])
def test_operands_and_results_in_columns_of_one_buffer(rows, left):
    """Rows that lie between one another share no element: codes beside values, results beside operands."""
    c, n = 64, 96
    buffer = torch.zeros(rows, 4 * c + n, dtype=torch.float16, device="cuda")
    values, result = (buffer[:, c:2 * c], buffer[:, :c]) if left else (buffer[:, :c], buffer[:, c:2 * c])
    values.normal_(generator=gen(50))
    x = values.clone()
    _, s = H.quantize_tokens(values, hb=32, codes="f16", out=result)
    finish()
    assert torch.equal(values, x)
    check_quantized(x, result, s, 32)
    w, one = codes(n, c, 51), torch.ones(max(n, rows), device="cuda")
    y = buffer[:, 2 * c:2 * c + n]
    H.linear(result, one[:rows].contiguous(), H.prepare_linear(w, scales=0.001 * one[:n]), out=y)
    finish()
    ref = integer_sums(result, w) * 0.001
    assert bool(((y.double() - ref).abs() <= (3.01 * 2.0 ** -24 + 1.01 * 2.0 ** -11) * ref.abs() + 2.0 ** -25).all())
    index = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0)[:, None].contiguous()
    H.combine_rows(values, index, one[:rows, None].contiguous(), out=result)
    finish()
    assert torch.equal(result, x.flip(0))
    H.combine_rows(values, index[:1].contiguous(), one[:1, None].contiguous(), out=result[rows // 2:rows // 2 + 1])
    finish()
    assert torch.equal(result[rows // 2], x[rows - 1])


def test_columns_that_share_an_element_are_refused():
    buffer = torch.zeros(40, 256, dtype=torch.float16, device="cuda")
    w, one = codes(96, 64, 52), torch.ones(96, device="cuda")
    L, index = H.prepare_linear(w, scales=one), torch.zeros(40, 1, dtype=torch.int32, device="cuda")
    s, x = one[:40].contiguous(), buffer[:, 96:160]
    for call in (lambda: H.quantize_tokens(x, out=buffer[:, 159:223], codes="f16"), lambda: H.quantize_tokens(x, out=buffer[:, 33:97], codes="f16"),
                 lambda: H.linear(x, s, L, out=buffer[:, 159:255]), lambda: H.linear(x, s, L, out=buffer[:, 1:97]),
                 lambda: H.combine_rows(x, index, s[:, None].contiguous(), out=buffer[:, 100:164]),
                 lambda: H.combine_rows(x, index, s[:, None].contiguous(), out=x),
                 lambda: H.combine_rows(x, index[:1].contiguous(), s[:1, None].contiguous(), out=buffer[3:4, 95:159])):
        with pytest.raises(H.HatqError):
            call()
    # the last row's end reaches into the buffer's next row
    wrapped = buffer.view(-1)[200:200 + 39 * 256].view(39, 256)[:, :64]
    with pytest.raises(H.HatqError):
        H.quantize_tokens(buffer[:39, :64], out=wrapped, codes="f16")
