"""Token operators on the GPU against plain formulas in 64 bits.

The products are compared exactly: with unit scales and float32 output the
result is the integer sum rounded once. Elsewhere the bounds follow from the
number of fp32 roundings, u = 2^-24 each, and one rounding to the output type.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# relative error of the one rounding to the output type: 0 (already fp32), 2^-11, 2^-8
HALF_ULP = {d: 0.0 if d == torch.float32 else torch.finfo(d).eps / 2 for d in TYPES.values()}
CODES = {"i8": torch.int8, "f16": torch.float16}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def codes(rows, k, seed, kind="i8", low=-127):
    return torch.randint(low, 128, (rows, k), generator=gen(seed), device="cuda").to(CODES[kind])


def integer_sums(x, w):
    """Exact: products below 2^14, at most 2^16 of them, in float64."""
    return x.double() @ w.double().T


def rand_scales(n, seed):
    return 0.01 * torch.exp(torch.randn(n, generator=gen(seed), device="cuda"))


def finish():
    torch.cuda.synchronize()
    H.sync_status()


# ------------------------------------------------------------------ linear

DENSE = [(1, 1, 1), (1, 64, 8), (1, 4096, 130), (2, 100, 77), (3, 1000, 129), (5, 17, 5), (7, 2047, 1000), (8, 512, 256),
         (9, 64, 128), (9, 1, 1), (16, 130, 40), (31, 4096, 257), (33, 999, 127), (48, 2048, 512), (64, 63, 300),
         (65, 320, 129), (127, 1024, 384), (128, 1025, 128), (129, 128, 640), (191, 640, 256), (193, 200, 1000),
         (225, 4160, 385), (300, 65, 2049), (777, 1000, 1234), (1000, 8192, 136)]


@pytest.mark.parametrize("rows,k,n", DENSE)
@pytest.mark.parametrize("kind", ["i8", "f16"])
def test_linear_sums_are_exact(rows, k, n, kind):
    x, w = codes(rows, k, 1, kind), codes(n, k, 2)
    one = torch.ones(max(rows, n), device="cuda")
    y = H.linear(x, one[:rows].contiguous(), H.prepare_linear(w, scales=one[:n]), dtype=torch.float32)
    finish()
    assert torch.equal(y, integer_sums(x, w).float())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,k,n,bias", [(1, 512, 100, True), (6, 130, 33, False), (40, 256, 130, True),
                                           (200, 1000, 300, False), (500, 320, 777, True)])
def test_linear_scales_bias_and_types(dtype, rows, k, n, bias):
    x, w = codes(rows, k, 3, "f16"), codes(n, k, 4)
    sx, sw = rand_scales(rows, 5), rand_scales(n, 6)
    b = torch.randn(n, generator=gen(7), device="cuda") if bias else None
    y = H.linear(x, sx, H.prepare_linear(w, scales=sw, bias=b), dtype=TYPES[dtype])
    finish()
    p = integer_sums(x, w) * sw.double() * sx.double()[:, None]
    ref = p if b is None else p + b.double()
    # conversion, two scales: 3 u of the product; the bias: u of the sum; the output type, and its subnormals
    tol = 3.01 * U * p.abs() + (1.01 * U + HALF_ULP[TYPES[dtype]] * 1.01) * ref.abs() + 2.0 ** -25
    assert y.dtype == TYPES[dtype] and bool(((y.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("rows", [4, 40, 130, 400])
@pytest.mark.parametrize("k", [1040, 5000, 20000])
def test_linear_past_the_exact_range_of_fp32(rows, k):
    """Sums far beyond 2^24 whose low bits matter: extreme codes, -128 among them, and a cancelling half."""
    x = torch.full((rows, k), 127, dtype=torch.float16, device="cuda")
    x[:, 1::2] = 126
    w = torch.full((136, k), 127, dtype=torch.int8, device="cuda")
    w[1] = -128
    w[2, k // 2:] = -127
    w[3] = codes(1, k, 8)[0]
    w[4, 5] = 126
    one = torch.ones(max(rows, 136), device="cuda")
    y = H.linear(x, one[:rows].contiguous(), H.prepare_linear(w, scales=one[:136]), dtype=torch.float32)
    finish()
    assert torch.equal(y, integer_sums(x, w).float())


def test_linear_windows_of_the_weights():
    """Bit j of an expert's word: some channel has an aligned window of 1024 << j codes with sum |w| > 2^17."""
    w = torch.zeros(4, 130, 5000, dtype=torch.int8, device="cuda")
    w[1, 129] = 64                      # 2048 * 64 = 2^17: allowed; 4096 codes of it are not
    w[2, 3, 1024:2048] = -128           # 2^17 alone, one more code next to it within 2048
    w[2, 3, 1023] = 1
    w[3, 7, :2000] = 100
    L = H.prepare_linear(w, scales=torch.ones(4, 130, device="cuda"))
    assert L.windows.tolist() == [0, 0b1111100, 0b1111110, 0b1111110]


@pytest.mark.parametrize("rows", [3, 50, 300])
def test_linear_strides_and_alignment(rows):
    k, n = 200, 150
    w, one = codes(n, k, 11), torch.ones(400, device="cuda")
    L = H.prepare_linear(w, scales=one[:n])
    for kind in CODES:
        wide = codes(2 * rows, k + 9, 12, kind)
        for x in (wide[::2, :k], wide[:rows, 1:k + 1], wide[:rows, 9:], wide[:1, :k].expand(rows, k)):
            big = torch.full((rows, n + 7), 5.0, device="cuda")
            out = big[:, 3:3 + n]
            H.linear(x, one[:rows].contiguous(), L, out=out)
            finish()
            assert torch.equal(out, integer_sums(x, w).float())
            assert bool((big[:, :3] == 5).all()) and bool((big[:, 3 + n:] == 5).all())


def test_linear_weights_from_strided_and_float_tensors():
    w = codes(64, 300, 13)
    one = torch.ones(64, device="cuda")
    x = codes(20, 200, 14, "f16")
    y = H.linear(x, one[:20].contiguous(), H.prepare_linear(w[:, 50:250], scales=one), dtype=torch.float32)
    z = H.linear(x, one[:20].contiguous(), H.prepare_linear(w.T.contiguous().T[:, 50:250], scales=one), dtype=torch.float32)
    finish()
    ref = integer_sums(x, w[:, 50:250]).float()
    assert torch.equal(y, ref) and torch.equal(z, ref)


@pytest.mark.parametrize("kind,k", [("i8", 2000), ("i8", 2001), ("f16", 2003), ("f16", 1024)])
def test_linear_of_many_rows_in_any_format(kind, k):
    rows, n = 3500, 4000
    x, w = codes(rows, k, 23, kind), codes(n, k, 24)
    one = torch.ones(n, device="cuda")
    L = H.prepare_linear(w, scales=one)
    y = H.linear(x, one[:rows].contiguous(), L, dtype=torch.float32)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    z = H.grouped_linear(x, one[:rows].contiguous(), off, H.prepare_linear(w[None], scales=one[None]), dtype=torch.float32)
    finish()
    ref = integer_sums(x, w).float()
    assert torch.equal(y, ref) and torch.equal(z, ref)


@pytest.mark.parametrize("rows", [2, 20, 150, 400])
def test_a_nan_scale_stays_in_its_row(rows):
    x, w = codes(rows, 128, 15, "f16"), codes(64, 128, 16)
    sx = torch.ones(rows, device="cuda")
    sx[1] = math.nan
    y = H.linear(x, sx, H.prepare_linear(w, scales=torch.ones(64, device="cuda")), dtype=torch.float32)
    finish()
    ref = integer_sums(x, w).float()
    assert bool(y[1].isnan().all())
    keep = torch.arange(rows, device="cuda") != 1
    assert torch.equal(y[keep], ref[keep])


@pytest.mark.parametrize("rows", [0, 1, 40])
def test_empty_and_half_precision_overflow(rows):
    x, w = codes(rows, 64, 17, "f16"), torch.full((10, 64), 127, dtype=torch.int8, device="cuda")
    x.fill_(127)
    y = H.linear(x, torch.ones(rows, device="cuda"), H.prepare_linear(w, scales=torch.ones(10, device="cuda")),
                 dtype=torch.float16)
    finish()
    assert y.shape == (rows, 10) and bool(y.isinf().all())


def test_linear_on_another_stream_and_in_a_graph():
    x, w = codes(100, 256, 18, "i8"), codes(200, 256, 19)
    one = torch.ones(200, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    L = H.prepare_linear(w, scales=one, stream=side)
    y = H.linear(x, one[:100].contiguous(), L, dtype=torch.float32, stream=side)
    side.synchronize()
    assert torch.equal(y, integer_sums(x, w).float())
    s, out = one[:100].contiguous(), torch.empty(100, 200, device="cuda")
    H.linear(x, s, L, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.linear(x, s, L, out=out)
    x.copy_(codes(100, 256, 20, "i8"))
    graph.replay()
    finish()
    assert torch.equal(out, integer_sums(x, w).float())


def test_linear_offsets_past_32_bits():
    rows, n, k = 140_000, 16_384, 64
    x, w = codes(rows, k, 21, "f16"), codes(n, k, 22)
    one = torch.ones(rows, device="cuda")
    y = H.linear(x, one, H.prepare_linear(w, scales=one[:n]), dtype=torch.bfloat16)
    finish()
    for r in (0, 131_071, 131_073, rows - 1):
        assert torch.equal(y[r], integer_sums(x[r:r + 1], w)[0].bfloat16())


@pytest.mark.parametrize("rows,k,n,kind", [(20, 2048, 512, "f16"), (60, 700, 300, "i8"), (600, 1024, 600, "f16"),
                                           (2000, 4096, 4096, "f16")])
def test_linear_behind_an_expired_wait(rows, k, n, kind):
    """A product enqueued behind a wait that ran out leaves its output alone; after the status was read all is as before."""
    x, w = codes(rows, k, 25, kind), codes(n, k, 26)
    one = torch.ones(max(rows, n), device="cuda")
    L, s = H.prepare_linear(w, scales=one[:n]), one[:rows].contiguous()
    finish()
    out = torch.full((rows, n), 3.0, device="cuda")
    H.selftest_wait(1000)
    H.linear(x, s, L, out=out)
    torch.cuda.synchronize()
    with pytest.raises(H.HatqError) as e:
        H.sync_status()
    assert e.value.status == H.ERR_TIMEOUT and bool((out == 3).all())
    H.linear(x, s, L, out=out)
    finish()
    assert torch.equal(out, integer_sums(x, w).float())


# ------------------------------------------------------------------ grouped_linear

def offsets_of(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")


def grouped_reference(x, w, off):
    y = torch.full((x.shape[0], w.shape[1]), math.nan, device="cuda")
    o = off.tolist()
    for e in range(w.shape[0]):
        if o[e + 1] > o[e]:
            y[o[e]:o[e + 1]] = integer_sums(x[o[e]:o[e + 1]], w[e]).float()
    return y


GROUPS = [[1], [0, 1, 0], [3, 0, 5], [8], [0, 0, 0, 0], [1] * 8, [2, 0, 1, 4, 0, 1], [5, 0, 11, 1], [40, 0, 0, 1], [32] * 5,
          [33, 31, 0, 64, 65, 1], [130, 0, 7, 128, 127, 129], [0, 300, 0, 0, 5, 191, 193, 0], [600, 1, 0, 250],
          [1] * 70 + [0] * 200 + [9] * 30, [0] * 1023 + [50]]


@pytest.mark.parametrize("counts", GROUPS, ids=lambda c: f"{len(c)}x{sum(c)}")
@pytest.mark.parametrize("k,n,kind", [(64, 128, "f16"), (300, 140, "i8"), (1100, 40, "f16")])
def test_grouped_sums_are_exact(counts, k, n, kind):
    rows, e = sum(counts), len(counts)
    x, w = codes(rows, k, 30, kind), codes(e * n, k, 31).view(e, n, k)
    off = offsets_of(counts)
    y = H.grouped_linear(x, torch.ones(rows, device="cuda"), off, H.prepare_linear(w, scales=torch.ones(e, n, device="cuda")),
                         dtype=torch.float32)
    finish()
    assert torch.equal(y, grouped_reference(x, w, off))


@pytest.mark.parametrize("rows,counts", [(8, [1, 2, 3]), (60, [20, 0, 15]), (900, [300, 200, 1])])
def test_rows_without_an_expert_are_left_alone(rows, counts):
    x, w = codes(rows, 128, 32, "f16"), codes(3 * 70, 128, 33).view(3, 70, 128)
    off = offsets_of(counts)
    x[sum(counts):] = math.nan                       # never read into a held row's result
    out = torch.full((rows, 70), -3.0, device="cuda")
    H.grouped_linear(x, torch.ones(rows, device="cuda"), off, H.prepare_linear(w, scales=torch.ones(3, 70, device="cuda")),
                     out=out)
    finish()
    held = sum(counts)
    assert torch.equal(out[:held], grouped_reference(x[:held], w, off))
    assert bool((out[held:] == -3).all())


@pytest.mark.parametrize("rows", [6, 50, 700])
def test_offsets_are_clamped_to_the_rows(rows):
    x, w = codes(rows, 64, 34, "f16"), codes(3 * 64, 64, 35).view(3, 64, 64)
    one = torch.ones(rows, device="cuda")
    L = H.prepare_linear(w, scales=torch.ones(3, 64, device="cuda"))
    wild = torch.tensor([-5, 2, rows + 100, rows + 7], dtype=torch.int32, device="cuda")
    y = H.grouped_linear(x, one, wild, L, dtype=torch.float32)
    finish()
    fine = torch.tensor([0, 2, rows, rows], dtype=torch.int32, device="cuda")
    assert torch.equal(y, grouped_reference(x, w, fine))


@pytest.mark.parametrize("rows", [7, 20, 60, 700])
def test_offsets_that_step_back(rows):
    """One below an earlier one counts as the earlier one: no row belongs to two experts."""
    e = 70
    x, w = codes(rows, 64, 41, "f16"), codes(e * 32, 64, 42).view(e, 32, 64)
    off = torch.randint(-3, rows + 3, (e + 1,), generator=gen(43), device="cuda", dtype=torch.int32)
    off[0], off[5], off[6], off[-1] = 1, rows // 2, 0, rows // 3
    fine = torch.cummax(off.clamp(0, rows), 0)[0]
    out = torch.full((rows, 32), -7.0, device="cuda")
    H.grouped_linear(x, torch.ones(rows, device="cuda"), off, H.prepare_linear(w, scales=torch.ones(e, 32, device="cuda")), out=out)
    finish()
    ref = grouped_reference(x, w, fine.int())
    held = ~ref[:, 0].isnan()
    assert bool(held.any()) and torch.equal(out[held], ref[held]) and bool((out[~held] == -7).all())


def test_grouped_scales_and_bias_belong_to_the_expert():
    counts, k, n = [3, 0, 90, 41], 192, 100
    rows = sum(counts)
    for r0 in (0, 3):
        c = counts if r0 == 0 else [1, 2, 0, 1]
        rows = sum(c)
        x, w = codes(rows, k, 36, "f16"), codes(4 * n, k, 37).view(4, n, k)
        sx, sw = rand_scales(rows, 38), rand_scales(4 * n, 39).view(4, n)
        b = torch.randn(4, n, generator=gen(40), device="cuda")
        off = offsets_of(c)
        y = H.grouped_linear(x, sx, off, H.prepare_linear(w, scales=sw, bias=b), dtype=torch.float32)
        finish()
        e = torch.repeat_interleave(torch.arange(4, device="cuda"), torch.tensor(c, device="cuda"))
        p = torch.einsum("rk,rnk->rn", x.double(), w.double()[e]) * sw.double()[e] * sx.double()[:, None]
        ref = p + b.double()[e]
        assert bool(((y.double() - ref).abs() <= 3.01 * U * p.abs() + 1.01 * U * ref.abs()).all())


@pytest.mark.parametrize("rows", [8, 100])
def test_grouped_weights_past_32_bits(rows):
    e, n, k = 40, 8192, 8192
    w = torch.empty(e, n, k, dtype=torch.int8, device="cuda")
    for i in range(e):
        w[i] = codes(n, k, 50 + i)
    counts = [0] * e
    counts[e - 1], counts[33] = rows - 2, 2
    x, off = codes(rows, k, 51, "f16"), offsets_of(counts)
    y = H.grouped_linear(x, torch.ones(rows, device="cuda"), off, H.prepare_linear(w, scales=torch.ones(e, n, device="cuda")),
                         dtype=torch.float32)
    finish()
    assert torch.equal(y[:2], integer_sums(x[:2], w[33]).float())
    assert torch.equal(y[2:], integer_sums(x[2:], w[e - 1]).float())


# ------------------------------------------------------------------ quantize_tokens

def act64(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "silu":
        return v * torch.sigmoid(v)
    return 0.5 * v * (1 + torch.erf(v / math.sqrt(2))) if act == "gelu" else v


def transform64(v, hb):
    i = np.arange(hb)
    h = torch.tensor([[1.0 - 2.0 * (bin(a & b).count("1") & 1) for b in i] for a in i], dtype=torch.float64, device="cuda")
    return (v.reshape(v.shape[0], -1, hb) @ h).reshape(v.shape)


def check_quantized(x, q, s, hb, act="none", gated=False, rows=None):
    """Codes within half a step of t * 127 / a, and the scales, up to fp32's roundings.

    Each value of u is off by at most 8 u |v w| (activation: expf or erff within 2 ulp, three operations; the
    gate's product), each transform stage adds u of the block's sum of magnitudes."""
    c = x.shape[1] // 2 if gated else x.shape[1]
    v = x.double()
    if rows is not None:
        r = rows.long()
        empty = (r < 0) | (r >= x.shape[0])
        v = torch.where(empty[:, None], 0.0, v[r.clamp(0, max(0, x.shape[0] - 1))])
    up = v[:, c:] if gated else torch.ones_like(v)
    u = act64(v[:, :c], act) * up
    off = 8 * U * (v[:, :c] * up).abs() if act != "none" or gated else torch.zeros_like(u)
    t = transform64(u, hb)
    blocks = lambda z: z.reshape(z.shape[0], -1, hb).sum(2).amax(1)
    err = math.log2(hb) * U * 1.01 * blocks(u.abs()) + blocks(off)
    a = t.abs().amax(1)
    zero = a == 0
    assert bool((s[zero] == 1).all()) and bool((q[zero] == 0).all())
    a, t, err, q, s = a[~zero], t[~zero], err[~zero], q[~zero].double(), s[~zero].double()
    step = torch.clamp(a / 127, min=2.0 ** -126)
    rel = err / a + 3.01 * U
    assert bool(((s - step / math.sqrt(hb)).abs() <= rel * s + 2.0 ** -149).all())
    z = t / step[:, None]
    assert bool((q.abs() <= 127).all())
    assert bool(((q - z).abs() <= 0.5 + 127 * (2 * rel)[:, None]).all())


SHAPES = [(1, 1, 1), (1, 8192, 256), (3, 7, 1), (5, 33, 1), (2, 34, 2), (17, 64, 64), (9, 96, 32), (40, 100, 4), (300, 200, 8),
          (31, 1000, 8), (33, 1024, 256), (12, 1056, 32), (7, 2000, 16), (64, 4096, 128), (3, 11008, 256), (2, 16384, 64),
          (2, 32768, 256), (1, 32767, 1)]


@pytest.mark.parametrize("rows,c,hb", SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", list(CODES))
def test_quantize(rows, c, hb, dtype, kind):
    x = (torch.randn(rows, c, generator=gen(60), device="cuda") * torch.exp(torch.randn(c, generator=gen(61), device="cuda")))
    x = x.to(TYPES[dtype])
    x[rows // 2] = 0
    q, s = H.quantize_tokens(x, hb=hb, codes=kind)
    finish()
    assert q.dtype == CODES[kind] and q.shape == (rows, c)
    check_quantized(x, q, s, hb)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,c,hb", [(1, 8192, 256), (50, 320, 64), (30, 99, 1), (6, 2000, 16)])
def test_quantize_activations(act, gated, rows, c, hb):
    for dtype in TYPES.values():
        x = (4 * torch.randn(rows, c * (1 + gated), generator=gen(62), device="cuda")).to(dtype)
        q, s = H.quantize_tokens(x, hb=hb, act=act, gated=gated)
        finish()
        check_quantized(x, q, s, hb, act, gated)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,c,hb", [(3, 32768, 256), (2, 9000, 8), (700, 8192, 128), (900, 2050, 2)])
def test_quantize_wide_gated_rows(dtype, rows, c, hb):
    x = torch.randn(rows, 2 * c, generator=gen(69), device="cuda").to(TYPES[dtype])
    q, s = H.quantize_tokens(x, hb=hb, act="silu", gated=True)
    finish()
    check_quantized(x, q, s, hb, "silu", True)


@pytest.mark.parametrize("rows,c,hb", [(20_000, 64, 64), (9_001, 200, 8), (5_000, 1000, 8), (3_001, 4096, 256), (2_000, 8192, 32),
                                       (500, 16384, 128)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_many_rows(rows, c, hb, dtype):
    """More rows than the GPU holds at once, gathered in part, a few of them empty or not finite."""
    x = torch.randn(rows, c, generator=gen(75), device="cuda").to(TYPES[dtype])
    x[7], x[rows - 2, 0] = 0, math.nan
    index = torch.randint(-1, rows + 1, (rows,), generator=gen(76), device="cuda").to(torch.int32)
    for at in (None, index):
        for kind in CODES:
            q, s = H.quantize_tokens(x, hb=hb, codes=kind, rows=at)
            finish()
            bad = s.isnan()
            source = torch.arange(rows, device="cuda") if at is None else at.long()
            assert torch.equal(bad, source == rows - 2) and bool((q[bad] == 0).all())
            keep = torch.where(~bad)[0]
            check_quantized(x, q[keep], s[keep], hb, rows=source[keep])


@pytest.mark.parametrize("gated", [False, True])
def test_quantize_gathers_rows(gated):
    x = torch.randn(50, 256 * (1 + gated), generator=gen(63), device="cuda").bfloat16()
    rows = torch.randint(-1, 51, (333,), generator=gen(64), device="cuda").to(torch.int32)
    rows[5], rows[6], rows[7] = -2 ** 31, 2 ** 31 - 1, 50
    q, s = H.quantize_tokens(x, hb=128, act="silu", gated=gated, rows=rows)
    finish()
    check_quantized(x, q, s, 128, "silu", gated, rows)
    q, s = H.quantize_tokens(x[:0], hb=128, gated=gated, rows=rows)
    finish()
    assert bool((q == 0).all()) and bool((s == 1).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_strides_and_alignment(dtype):
    wide = torch.randn(40, 531, generator=gen(65), device="cuda").to(TYPES[dtype])
    for x in (wide[::2, :512], wide[:, 1:513], wide[:, 19:], wide[:1, :512].expand(9, 512)):
        for kind in CODES:
            big = torch.full((x.shape[0], 520), 99, dtype=CODES[kind], device="cuda")
            out = big[:, 5:517]
            _, s = H.quantize_tokens(x, hb=32, codes=kind, out=out)
            finish()
            check_quantized(x, out, s, 32)
            assert bool((big[:, :5] == 99).all()) and bool((big[:, 517:] == 99).all())


@pytest.mark.parametrize("c,hb", [(64, 1), (64, 32), (4096, 128)])
@pytest.mark.parametrize("kind", list(CODES))
def test_quantize_special_rows(c, hb, kind):
    x = torch.randn(8, c, generator=gen(66), device="cuda")
    x[1, 3], x[2, 5], x[3, 0] = math.nan, math.inf, -math.inf
    x[4] = 0
    x[5] *= 1e-44                          # subnormal, most of it zero
    x[6] *= 1e37
    q, s = H.quantize_tokens(x, hb=hb, codes=kind)
    finish()
    assert bool(s[1:4].isnan().all()) and bool((q[1:4] == 0).all())
    rest = torch.tensor([0, 4, 5, 7] + ([6] if hb == 1 else []), device="cuda")
    check_quantized(x[rest], q[rest], s[rest], hb)


def test_quantize_ties_round_to_even():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    q, s = H.quantize_tokens(x, codes="i8")
    finish()
    assert q[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126] and s.tolist() == [1.0]


def test_quantize_offsets_past_32_bits():
    x = torch.empty(70_000, 32768, dtype=torch.bfloat16, device="cuda")
    x[65_530:65_545].normal_(generator=gen(67))
    x[-1].normal_(generator=gen(68))
    q, s = H.quantize_tokens(x, hb=64, codes="f16")
    finish()
    for r in (slice(65_530, 65_545), slice(69_999, 70_000)):
        check_quantized(x[r], q[r], s[r], 64)


# ------------------------------------------------------------------ combine_rows

@pytest.mark.parametrize("tokens,topk,c", [(1, 1, 1), (1, 8, 2048), (32, 8, 2048), (7, 3, 33), (100, 2, 1000), (5, 64, 8),
                                           (1000, 6, 320)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_combine(tokens, topk, c, dtype):
    y = torch.randn(tokens * topk + 3, c, generator=gen(70), device="cuda").to(TYPES[dtype])
    index = torch.randint(-1, tokens * topk + 4, (tokens, topk), generator=gen(71), device="cuda").to(torch.int32)
    weights = torch.rand(tokens, topk, generator=gen(72), device="cuda")
    if tokens > 2:
        index[1] = -1                       # a token that no expert kept
        index[2, 0] = 2 ** 31 - 1
    y[0] = math.inf if tokens == 7 else y[0]
    index[index == 0] = -1                  # so that the infinite row is not taken
    out = H.combine_rows(y, index, weights)
    finish()
    i = index.long()
    valid = (i >= 0) & (i < y.shape[0])
    z = torch.where(valid[:, :, None], y.double()[i.clamp(0, y.shape[0] - 1)] * weights.double()[:, :, None], 0.0)
    ref = z.sum(1)
    tol = (topk + 1) * 1.01 * U * z.abs().sum(1) + HALF_ULP[TYPES[dtype]] * 1.01 * ref.abs() + 2.0 ** -25
    assert bool(((out.double() - ref).abs() <= tol).all())
    if tokens > 2:
        assert bool((out[1] == 0).all())


@pytest.mark.parametrize("topk", [2, 4, 8, 12])
@pytest.mark.parametrize("c", [6, 34, 256, 1030])
def test_combine_off_the_usual_boundaries(topk, c):
    """Rows on 4-byte boundaries, and indices and weights that begin off 16-byte ones."""
    tokens = 50
    index = torch.randint(-1, 90, (tokens * topk + 1,), generator=gen(77), device="cuda").to(torch.int32)[1:].view(tokens, topk)
    weights = torch.rand(tokens * topk + 1, generator=gen(78), device="cuda")[1:].view(tokens, topk)
    for dtype in TYPES.values():
        y = torch.randn(88, c, generator=gen(79), device="cuda").to(dtype)
        out = H.combine_rows(y, index, weights)
        finish()
        i = index.long()
        valid = (i >= 0) & (i < 88)
        z = torch.where(valid[:, :, None], y.double()[i.clamp(0, 87)] * weights.double()[:, :, None], 0.0)
        ref = z.sum(1)
        tol = (topk + 1) * 1.01 * U * z.abs().sum(1) + HALF_ULP[dtype] * 1.01 * ref.abs() + 2.0 ** -25
        assert bool(((out.double() - ref).abs() <= tol).all())


def test_combine_strides():
    wide = torch.randn(60, 211, generator=gen(73), device="cuda").half()
    index = torch.randint(0, 30, (20, 2), generator=gen(74), device="cuda").to(torch.int32)
    weights = torch.ones(20, 2, device="cuda")
    for y in (wide[::2, :200], wide[:30, 3:203], wide[:1, :200].expand(30, 200)):
        big = torch.full((20, 207), 9.0, dtype=torch.float16, device="cuda")
        H.combine_rows(y, index, weights, out=big[:, 1:201])
        finish()
        i = index.long()
        assert torch.equal(big[:, 1:201], (y[i[:, 0]].float() + y[i[:, 1]].float()).half())
        assert bool((big[:, :1] == 9).all()) and bool((big[:, 201:] == 9).all())


# ------------------------------------------------------------------ together

def test_float_weights_follow_the_float_layer():
    """Quantized end to end against the float layer: the codes' steps bound the difference.

    Each operand is off by at most half a step per value (s_x / 2, s_w / 2 plus rounding), so by Cauchy-Schwarz
    |y - ref| <= sqrt(k) (s_x |w| + s_w |x|) / 2 + k s_x s_w / 4 up to fp32 roundings, the transform orthogonal."""
    for rows in (4, 200):
        x = torch.randn(rows, 512, generator=gen(80), device="cuda")
        w = torch.randn(300, 512, generator=gen(81), device="cuda") * 0.05
        L = H.prepare_linear(w, hb=128)
        q, s = H.quantize_tokens(x, hb=128)
        y = H.linear(q, s, L, dtype=torch.float32)
        finish()
        ref = x.double() @ w.double().T
        sx, sw, k = s.double()[:, None], L.s_w.double()[None], 512
        bound = math.sqrt(k) * (sx * w.double().norm(dim=1)[None] + sw * x.double().norm(dim=1)[:, None]) / 2 + k * sx * sw / 4
        assert bool(((y.double() - ref).abs() <= 1.001 * bound).all())
        assert float((y - ref).norm() / ref.norm()) < 0.05


# ------------------------------------------------------------------ refusals of the binding

def test_binding_refuses():
    x, w = codes(4, 64, 90), codes(32, 64, 91)
    one = torch.ones(64, device="cuda")
    L = H.prepare_linear(w, scales=one[:32])
    G = H.prepare_linear(w.view(2, 16, 64), scales=one[:32].view(2, 16))
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    s = one[:4].contiguous()
    bad = [lambda: H.linear(x.float(), s, L), lambda: H.linear(x[:, :32], s, L), lambda: H.linear(x.T, s, L),
           lambda: H.linear(x.cpu(), s, L), lambda: H.linear(x, one, L), lambda: H.linear(x, s.double(), L),
           lambda: H.linear(x, s.cpu(), L), lambda: H.linear(x, s, L, dtype=torch.float64), lambda: H.linear(x, s, G),
           lambda: H.linear(x, s, L, out=torch.empty(4, 31, device="cuda")),
           lambda: H.linear(x, s, L, out=torch.empty(1, 32, device="cuda").expand(4, 32)),
           lambda: H.linear(x, s, L, out=torch.empty(32, 4, device="cuda").T),
           lambda: H.grouped_linear(x, s, None, G), lambda: H.grouped_linear(x, s, off[:2], G),
           lambda: H.grouped_linear(x, s, off.long(), G), lambda: H.prepare_linear(w), lambda: H.prepare_linear(w, hb=2, scales=one[:32]),
           lambda: H.prepare_linear(w, scales=one), lambda: H.prepare_linear(w.half(), scales=one[:32]),
           lambda: H.prepare_linear(w[0], scales=one[:32]), lambda: H.prepare_linear(w, scales=one[:32], bias=one),
           lambda: H.quantize_tokens(x), lambda: H.quantize_tokens(x.half(), act="tanh"), lambda: H.quantize_tokens(x.half(), codes="i4"),
           lambda: H.quantize_tokens(x.half()[:, :63], gated=True), lambda: H.quantize_tokens(x.half(), rows=off.long()),
           lambda: H.quantize_tokens(x.half(), codes="i8", out=torch.empty(4, 64, dtype=torch.float16, device="cuda")),
           lambda: H.quantize_tokens(x.half(), scales=one), lambda: H.combine_rows(x, off.view(1, 3), one[:3].view(1, 3)),
           lambda: H.combine_rows(x.half(), off.view(1, 3), one[:2].view(1, 2)), lambda: H.combine_rows(x.half(), off, one[:3]),
           lambda: H.combine_rows(x.half(), off.view(1, 3), one[:3].contiguous().view(1, 3), out=torch.empty(1, 64, device="cuda"))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")
    for call in (lambda: H.quantize_tokens(x.half(), hb=3), lambda: H.quantize_tokens(x.half(), hb=128),
                 lambda: H.prepare_linear(w.half(), hb=48)):
        with pytest.raises(H.HatqError):
            call()
    finish()
