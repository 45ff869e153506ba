"""Products with 4-bit weights on the GPU against plain formulas.

With whole numbers for x and powers of two for the scales every sum is exact in
fp32, and the result is compared bit for bit. Elsewhere the bounds count the
roundings, u = 2^-24 each.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INF, NAN = math.inf, math.nan


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def finish():
    torch.cuda.synchronize()
    H.sync_status()


def codes(n, k, seed):
    return torch.randint(-8, 8, (n, k), generator=gen(seed), device="cuda").to(torch.int8)


def whole(rows, k, seed, dtype, most=8):
    return torch.randint(-most, most + 1, (rows, k), generator=gen(seed), device="cuda").to(dtype)


def formula(x, w, s, group, sx=None, bias=None):
    """In 64 bits: the result, and the sum of the terms' magnitudes."""
    m = w.double() * torch.repeat_interleave(s.double(), group, 1)[:, :w.shape[1]]
    f = 1 if sx is None else sx.double()[:, None]
    y = x.double() @ m.T * f
    return y if bias is None else y + bias.double(), x.double().abs() @ m.abs().T * (f if sx is None else f.abs())


SIZES = [(1, 1, 1), (1, 64, 16), (1, 4096, 130), (2, 100, 77), (3, 1000, 129), (5, 17, 5), (7, 2047, 1000), (8, 512, 256), (8, 63, 15),
         (9, 64, 128), (9, 33, 17), (16, 130, 40), (17, 4096, 257), (31, 65, 127), (32, 999, 300), (33, 2048, 512), (48, 640, 100),
         (63, 128, 33), (64, 300, 64), (65, 320, 129), (129, 1025, 128), (200, 512, 1000)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("group", [32, 64, 96, 128, 1024])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_whole_numbers_are_exact(rows, k, n, group, dtype):
    x, w = whole(rows, k, 1, TYPES[dtype]), codes(n, k, 2)
    s = 2.0 ** torch.randint(-1, 2, (n, -(-k // group)), generator=gen(3), device="cuda")
    y = H.linear4(x, H.prepare_linear4(w, group, scales=s), dtype=torch.float32)
    finish()
    assert torch.equal(y.double(), formula(x, w, s, group)[0])


def test_single_precision_inputs_are_whole():
    """Values of more bits than a 16-bit type holds: sums below 2^24 of their last places are exact."""
    x, w = whole(6, 500, 1, torch.float32, 4000), codes(100, 500, 2)
    x[:, 3] = 8_000_001
    w[:, 3] = torch.arange(100, device="cuda").remainder(2).to(torch.int8)
    x[:, 64:] = 0
    s = torch.ones(100, 4, device="cuda")
    y = H.linear4(x, H.prepare_linear4(w, 128, scales=s))
    finish()
    assert y.dtype == torch.float32 and torch.equal(y.double(), formula(x, w, s, 128)[0])


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,k,n,group,bias", [(1, 512, 100, 64, True), (6, 130, 33, 32, False), (12, 1000, 130, 128, True),
                                                 (40, 4096, 300, 32, False), (64, 320, 77, 128, True)])
def test_scales_bias_and_types(dtype, out, rows, k, n, group, bias):
    x = (torch.randn(rows, k, generator=gen(1), device="cuda") * torch.exp(torch.randn(k, generator=gen(2), device="cuda"))).to(TYPES[dtype])
    w = codes(n, k, 3)
    s = 0.01 * torch.exp(torch.randn(n, -(-k // group), generator=gen(4), device="cuda"))
    sx = torch.exp(torch.randn(rows, generator=gen(5), device="cuda"))
    b = torch.randn(n, generator=gen(6), device="cuda") if bias else None
    y = H.linear4(x, H.prepare_linear4(w, group, scales=s, bias=b), scales=sx, dtype=TYPES[out])
    finish()
    ref, terms = formula(x, w, s, group, sx, b)
    # a step's 17 terms, each cut to 24 bits of the largest, 4 steps (single precision: three times as many) before a
    # sum is scaled; then a rounding per block of 64 (two with small groups) and per joined warp, the scale of the row
    parts = 3 if dtype == "f32" else 1
    tol = U * (17 * 4 * parts + 2 * -(-k // 64) / 8 + 8 + 2) * terms + (U + (torch.finfo(TYPES[out]).eps / 2)) * 1.01 * ref.abs() + 2.0 ** -24
    assert y.dtype == TYPES[out] and float(((y.double() - ref).abs() / tol).max()) <= 1


def test_large_and_small_values():
    """The whole range of the inputs' types goes through: nothing is scaled on the way in."""
    for dtype, big, small in ((torch.bfloat16, 1e37, 1e-30), (torch.float16, 60000.0, 1e-7), (torch.float32, 1e37, 1e-30)):
        x = torch.zeros(3, 128, dtype=dtype, device="cuda")
        x[0, 5], x[1, 7], x[2, 100] = big, small, -big
        w = codes(20, 128, 1)
        w[:, 5], w[:, 7], w[:, 100] = 7, -8, 3
        y = H.linear4(x, H.prepare_linear4(w, 64, scales=torch.full((20, 2), 0.5, device="cuda")), dtype=torch.float32)
        finish()
        want = torch.stack([x[0, 5].double() * 3.5, x[1, 7].double() * -4, x[2, 100].double() * 1.5])[:, None]
        # 16-bit values: products of 11 + 3 bits, exact. Single precision: 7 x has 27 bits. Its three parts are added from
        # the smallest on, each sum cut to 24 bits of its largest term: by less than 2^-23 of the result in the last
        # step, of 2^-8 and 2^-16 of it before; the scale is a power of two. Below (1 + 2^-8 + 2^-16) 2^-23 together.
        tol = 2.0 ** -23 * 1.01 if dtype == torch.float32 else 0.0
        assert bool(((y.double() - want).abs() <= tol * want.abs()).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_infinities_and_nans_stay_in_their_row(dtype):
    x = whole(20, 200, 1, TYPES[dtype])
    w = codes(40, 200, 2)
    w[w == 0] = 1
    L = H.prepare_linear4(w, 32, scales=torch.ones(40, 7, device="cuda"))
    want = H.linear4(x, L, dtype=torch.float32)
    x[3, 7], x[9, 150], x[19, 199] = INF, NAN, -INF
    y = H.linear4(x, L, dtype=torch.float32)
    finish()
    assert torch.equal(y[3], w[:, 7].float() * INF) and torch.equal(y[19], w[:, 199].float() * -INF) and bool(y[9].isnan().all())
    keep = [r for r in range(20) if r not in (3, 9, 19)]
    assert torch.equal(y[keep], want[keep])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [1, 6, 20, 50])
def test_strides(dtype, rows):
    """Columns of a buffer, an odd pitch, one row for all, an output between other columns: nothing else is written."""
    k, n = 200, 70
    w, s = codes(n, k, 2), torch.ones(n, 2, device="cuda")
    L = H.prepare_linear4(w, 128, scales=s)
    wide = whole(rows, 3 * k + 1, 1, TYPES[dtype])
    for x in (wide[:, k:2 * k], wide[:, 1:k + 1], whole(1, k, 3, TYPES[dtype]).expand(rows, k)):
        out = torch.full((rows, n + 9), 7.0, dtype=torch.float32, device="cuda")
        got = H.linear4(x, L, out=out[:, 5:5 + n])
        finish()
        assert torch.equal(got.double(), formula(x, w, s, 128)[0])
        assert bool((out[:, :5] == 7).all()) and bool((out[:, 5 + n:] == 7).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("hb,k", [(1, 200), (2, 330), (32, 32), (64, 448), (128, 1024), (256, 4096)])
@pytest.mark.parametrize("group", [32, 128])
def test_quantize_groups_is_the_formula(dtype, hb, k, group):
    """Codes and scales in single precision, bit for bit; then the product with codes of tokens in the same basis."""
    w = torch.randn(37, k, generator=gen(1), device="cuda").to(TYPES[dtype])
    w[5], w[6, :3] = 0, 0
    c, s = H.quantize_groups(w, group, hb)
    finish()
    t, h = w.float().cpu().numpy(), 1
    while h < hb:
        t = t.reshape(37, -1, 2, h)
        t = np.stack([t[:, :, 0] + t[:, :, 1], t[:, :, 0] - t[:, :, 1]], 2).reshape(37, k)
        h *= 2
    inv = np.float32(1 / math.sqrt(hb))
    for g in range(-(-k // group)):
        part = t[:, g * group:(g + 1) * group]
        a = np.abs(part).max(1, keepdims=True)
        want = np.where(a > 0, np.rint(np.float32(7) * part / np.where(a > 0, a, 1)), 0)
        assert np.array_equal(c[:, g * group:(g + 1) * group].cpu().numpy(), want)
        assert np.array_equal(s[:, g].cpu().numpy(), np.where(a > 0, a / np.float32(7), np.float32(1))[:, 0] * inv)
    L = H.prepare_linear4(w, group, hb)
    x = torch.randn(9, k, generator=gen(2), device="cuda").to(TYPES[dtype])
    q, sx = H.quantize_tokens(x, hb=hb, codes="f16")
    y = H.linear4(q, L, scales=sx, dtype=torch.float32)
    finish()
    ref, terms = formula(q, c, s, group, sx)
    assert bool(((y.double() - ref).abs() <= U * (17 * 4 + 2 * k / 64 / 8 + 12) * terms + U * ref.abs()).all())


def test_quantize_groups_without_a_scale():
    w = torch.randn(4, 64, generator=gen(1), device="cuda")
    w[0, 5], w[1, 40], w[2, 0] = INF, NAN, 3e38
    c, s = H.quantize_groups(w, 32)
    finish()
    bad = torch.tensor([[1, 0], [0, 1], [1, 0], [0, 0]], dtype=torch.bool, device="cuda")
    assert torch.equal(s.isnan(), bad) and bool((c.reshape(4, 2, 32)[bad] == 0).all()) and bool((c.reshape(4, 2, 32)[~bad] != 0).any())


def test_codes_are_clamped_and_inputs_kept():
    w = torch.arange(-128, 128, device="cuda").to(torch.int8).repeat(16, 1)
    s = torch.ones(16, 2, device="cuda")
    L = H.prepare_linear4(w, 128, scales=s)
    y = H.linear4(torch.eye(256, device="cuda").bfloat16(), L, dtype=torch.float32)
    finish()
    assert torch.equal(y, w.T.float().clamp(-8, 7))


def test_in_a_graph_and_on_two_streams():
    w, s = codes(300, 1000, 2), torch.ones(300, 8, device="cuda")
    L = H.prepare_linear4(w, 128, scales=s)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    x, z = whole(5, 1000, 3, torch.float16), whole(30, 1000, 4, torch.bfloat16)
    torch.cuda.synchronize()
    got = [(H.linear4(x, L, stream=a, dtype=torch.float32), H.linear4(z, L, stream=b, dtype=torch.float32)) for _ in range(10)]
    finish()
    for y, u in got:
        assert torch.equal(y.double(), formula(x, w, s, 128)[0]) and torch.equal(u.double(), formula(z, w, s, 128)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = H.linear4(x, L, dtype=torch.float32)
    for seed in (7, 8):
        x.copy_(whole(5, 1000, seed, torch.float16))
        graph.replay()
        finish()
        assert torch.equal(y.double(), formula(x, w, s, 128)[0])


def test_refusals():
    w, s = codes(30, 100, 1), torch.ones(30, 1, device="cuda")
    L = H.prepare_linear4(w, 128, scales=s)
    x = whole(3, 100, 2, torch.float16)
    for bad in (lambda: H.linear4(x[:, :99], L), lambda: H.linear4(x.double(), L), lambda: H.linear4(x.cpu(), L), lambda: H.linear4(x[0], L),
                lambda: H.linear4(x, L, dtype=torch.int8), lambda: H.linear4(x, L, scales=torch.ones(2, device="cuda")),
                lambda: H.linear4(x, L, out=torch.empty(3, 29, device="cuda")), lambda: H.prepare_linear4(w, 128),
                lambda: H.prepare_linear4(w, 32, scales=s), lambda: H.prepare_linear4(w, 100, scales=s),
                lambda: H.prepare_linear4(w.float(), 128, scales=s), lambda: H.prepare_linear4(w.float(), 128, hb=8),
                lambda: H.prepare_linear4(w, 128, scales=s, bias=torch.ones(29)), lambda: H.prepare_linear4(w[0], 128, scales=s),
                lambda: H.quantize_groups(w.float(), 31), lambda: H.quantize_groups(w, 32)):
        with pytest.raises((ValueError, H.HatqError)):
            bad()
    finish()


@pytest.mark.parametrize("group", [2 ** 31 - 32, 2 ** 31 - 128])
def test_the_largest_groups(group):
    """One scale a channel, the group's size as large as an int allows: as with a group of all inputs."""
    w = torch.randn(37, 320, generator=gen(1), device="cuda")
    c, s = H.quantize_groups(w, group, 64)
    want = H.quantize_groups(w, 320, 64)
    x = whole(3, 320, 2, torch.bfloat16)
    y = H.linear4(x, H.prepare_linear4(w, group, 64), dtype=torch.float32)
    finish()
    assert c.shape == (37, 320) and s.shape == (37, 1) and torch.equal(c, want[0]) and torch.equal(s, want[1])
    ref, terms = formula(x, c, s, 320)
    assert bool(((y.double() - ref).abs() <= U * (17 * 4 + 2 * 5 / 8 + 12) * terms + U * ref.abs()).all())


@pytest.mark.parametrize("rows", [5, 40])
def test_any_nan_in_single_precision_is_one(rows):
    """NaNs whose upper 16 bits are those of an infinity among them."""
    x = whole(rows, 200, 1, torch.float32)
    w = codes(40, 200, 2)
    w[w == 0] = 1
    L = H.prepare_linear4(w, 32, scales=torch.ones(40, 7, device="cuda"))
    want = H.linear4(x, L)
    bits = torch.tensor([0x7f800001, 0x7f80ffff, -0x7fffff, 0x7fffffff], dtype=torch.int32, device="cuda").view(torch.float32)
    for r in range(4):
        x[r, 50 * r] = bits[r]
    y = H.linear4(x, L)
    finish()
    assert bool(y[:4].isnan().all()) and torch.equal(y[4:], want[4:])
