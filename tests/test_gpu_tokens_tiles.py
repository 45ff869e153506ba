"""Products on every tile, split and operand form of the tensor-core kernel and every form of the dot-product kernel, exactly.

Each case names the kernel it is meant for and checks that the library takes it. Unit scales and float32 output give the
integer sum rounded once; the 16-bit types round that once more. The weights hold channels of extreme codes, so sums past
the exact range of fp32 come in several windows wherever the reduction is longer than 1024.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H
from tests.test_gpu_tokens import CODES, codes, finish, grouped_reference, integer_sums, offsets_of

pytestmark = pytest.mark.gpu

# tokens per tile, CTAs per tile, CTAs per reduction; rows, k, n
DENSE = [((32, 1, 1), 20, 200, 130), ((32, 1, 1), 20, 5000, 19400), ((32, 1, 2), 20, 5000, 9000), ((32, 1, 4), 20, 5000, 130),
         ((64, 1, 1), 33, 5000, 19400), ((64, 1, 1), 2500, 200, 130), ((64, 1, 2), 33, 5000, 9000), ((64, 1, 4), 777, 5000, 130),
         ((128, 1, 1), 6000, 200, 300), ((128, 1, 2), 2500, 5000, 130), ((128, 1, 4), 1300, 5000, 130),
         ((128, 2, 1), 6000, 200, 130), ((128, 2, 1), 6389, 5000, 130), ((192, 2, 1), 2500, 200, 1000),
         ((192, 2, 1), 130, 5000, 19400)]
GROUPED = [((32, 1, 1), 33, 5000, 1500), ((32, 1, 2), 33, 5000, 700), ((32, 1, 4), 33, 5000, 130), ((64, 1, 1), 200, 5000, 2100),
           ((64, 1, 2), 300, 5000, 700), ((64, 1, 4), 500, 5000, 130), ((128, 1, 1), 6000, 200, 300), ((128, 1, 2), 2500, 5000, 130),
           ((128, 1, 4), 1300, 5000, 130), ((128, 2, 1), 6000, 200, 130), ((128, 2, 1), 6389, 5000, 130),
           ((192, 2, 1), 700, 200, 2100), ((192, 2, 1), 777, 5000, 2100)]
LOOSE_DENSE = [((32, 1, 1), 20, 200, 130), ((32, 1, 2), 20, 5000, 9000), ((32, 1, 4), 20, 5000, 130), ((64, 1, 1), 2500, 200, 130),
               ((64, 1, 2), 33, 5000, 9000), ((64, 1, 4), 777, 5000, 130), ((128, 1, 1), 6389, 5000, 130),
               ((128, 1, 2), 2500, 5000, 130), ((128, 1, 4), 1300, 5000, 130)]
LOOSE_GROUPED = [((32, 1, 1), 33, 5000, 1500), ((32, 1, 2), 33, 5000, 700), ((32, 1, 4), 33, 5000, 130), ((64, 1, 1), 200, 5000, 2100),
                 ((64, 1, 2), 300, 5000, 700), ((64, 1, 4), 500, 5000, 130), ((128, 1, 1), 6389, 5000, 130),
                 ((128, 1, 2), 2500, 5000, 130), ((128, 1, 4), 1300, 5000, 130)]
PACKED_DENSE = [((32, 1, 1), 20, 5000, 19400), ((64, 1, 2), 33, 5000, 9000), ((128, 1, 2), 130, 5000, 3970),
                ((128, 1, 4), 130, 5000, 1500), ((128, 2, 1), 777, 5000, 1500), ((192, 2, 1), 130, 5000, 19400)]
PACKED_GROUPED = [((32, 1, 2), 33, 5000, 700), ((64, 1, 1), 200, 5000, 2100), ((128, 1, 2), 777, 5000, 700),
                  ((128, 2, 1), 500, 5000, 2100), ((192, 2, 1), 777, 5000, 2100)]
# the dot-product kernel: rows per pass; rows, k, n. A reduction of up to 2048 and many channels: two per thread
FEW_DENSE = [(1, 1, 4096, 130), (1, 1, 2048, 4870), (1, 1, 65, 5001), (2, 2, 5000, 130), (2, 2, 1000, 4899), (4, 3, 300, 130),
             (4, 4, 5000, 4870), (8, 5, 64, 200), (8, 8, 3000, 2000)]
FEW_GROUPED = [(1, 8, 5000, 130), (1, 24, 2048, 203), (1, 24, 65, 5001), (1, 13, 1000, 700)]
EXPERTS = 8


def operand(rows, k, kind, pad, seed):
    """Codes at a pitch of k + pad, beginning pad elements in where rows are not to lie on 16-byte boundaries."""
    wide = torch.zeros(rows, k + 2 * pad, dtype=CODES[kind], device="cuda")
    x = wide[:, pad:pad + k] if pad else wide
    x.copy_(codes(rows, k, seed, kind, -128))
    x[0], x[rows // 2], x[rows - 1] = 127, -128, 126
    return x


def weight_codes(experts, n, k, seed):
    w = codes(experts * n, k, seed, "i8", -128).view(experts, n, k)
    w[:, 0], w[:, 1] = 127, -128
    w[:, n // 2, k // 2:] = -127
    w[:, n - 1] = 127
    return w


def ragged(rows):
    """Rows per expert: idle ones, one row, one less and one more than a tile's columns, the rest on three experts."""
    counts = [0, 1, 0, 31 if rows > 128 else 3, 33 if rows > 128 else 5]
    if rows > 1000:
        counts[2], counts[4] = 191, 193
    left = rows - sum(counts)
    return counts + [left - left // 3 - left // 7, left // 7, left // 3]


def check(tile, rows, k, n, kind, pad, grouped, way, few=False):
    e = EXPERTS if grouped else 1
    counts = ([0, 1, rows - 4, 0, 0, 3, 0, 0] if few else ragged(rows)) if grouped else [rows]
    extra = 3 if grouped else 0                      # rows that no expert holds
    x, w = operand(rows + extra, k, kind, pad, rows), weight_codes(e, n, k, n)
    off = offsets_of(counts) if grouped else None
    one = torch.ones(max(rows + extra, n), device="cuda")
    L = H.prepare_linear(w if grouped else w[0], scales=one[:n].repeat(e, 1) if grouped else one[:n])
    ref = grouped_reference(x, w, off)[:rows] if grouped else integer_sums(x, w[0]).float()
    lib, fmt, raw = H.load(), H.CODES_I8 if kind == "i8" else H.CODES_F16, torch.cuda.current_stream().cuda_stream
    space = torch.empty(2 * (rows + extra) * -(-k // 64) * 64 if way == 2 else 0, dtype=torch.uint8, device="cuda")
    plan = (ctypes.c_int * 5)()
    assert lib.hatq_linear_plan(x.data_ptr(), fmt, x.stride(0), rows + extra, L.ref, int(grouped), space.numel(), plan) == H.OK
    assert list(plan) == [int(few), *tile, way]
    for dtype, code, gap in ((torch.float32, H.F32, 0), (torch.bfloat16, H.BF16, 0), (torch.bfloat16, H.BF16, 1),
                             (torch.float16, H.F16, 2)):
        y = torch.full((rows + extra, n + gap), 7.0, dtype=dtype, device="cuda")
        args = (y.data_ptr(), y.stride(0), space.data_ptr() if way == 2 else None, space.numel(), raw)
        if grouped:
            st = lib.hatq_grouped_linear(x.data_ptr(), fmt, x.stride(0), one.data_ptr(), rows + extra, off.data_ptr(), L.ref, code,
                                         *args)
        else:
            st = lib.hatq_linear(x.data_ptr(), fmt, x.stride(0), one.data_ptr(), rows, L.ref, code, *args)
        assert st == H.OK, H.last_error()
        finish()
        assert torch.equal(y[:rows, :n], ref.to(dtype))
        assert bool((y[rows:] == 7).all()) and bool((y[:, n:] == 7).all())


def name(v):
    return "x".join(map(str, v)) if isinstance(v, tuple) else None


@pytest.mark.parametrize("tile,rows,k,n", DENSE, ids=name)
def test_dense_tiles(tile, rows, k, n):
    check(tile, rows, k, n, "f16", 0, False, 0)


@pytest.mark.parametrize("tile,rows,k,n", GROUPED, ids=name)
def test_grouped_tiles(tile, rows, k, n):
    check(tile, rows - 3, k, n, "f16", 0, True, 0)


@pytest.mark.parametrize("kind,pad", [("i8", 0), ("i8", 1), ("i8", 4), ("i8", 8), ("f16", 1), ("f16", 2)])
@pytest.mark.parametrize("tile,rows,k,n", LOOSE_DENSE, ids=name)
def test_dense_tiles_of_codes_as_they_lie(tile, rows, k, n, kind, pad):
    check(tile, rows, k, n, kind, pad, False, 1)


@pytest.mark.parametrize("kind,pad", [("i8", 0), ("i8", 1), ("f16", 1)])
@pytest.mark.parametrize("tile,rows,k,n", LOOSE_GROUPED, ids=name)
def test_grouped_tiles_of_codes_as_they_lie(tile, rows, k, n, kind, pad):
    check(tile, rows - 3, k, n, kind, pad, True, 1)


@pytest.mark.parametrize("kind,pad", [("i8", 0), ("f16", 1)])
@pytest.mark.parametrize("tile,rows,k,n", PACKED_DENSE, ids=name)
def test_dense_tiles_of_packed_codes(tile, rows, k, n, kind, pad):
    check(tile, rows, k, n, kind, pad, False, 2)


@pytest.mark.parametrize("kind,pad", [("i8", 1), ("f16", 1)])
@pytest.mark.parametrize("tile,rows,k,n", PACKED_GROUPED, ids=name)
def test_grouped_tiles_of_packed_codes(tile, rows, k, n, kind, pad):
    check(tile, rows - 3, k, n, kind, pad, True, 2)


@pytest.mark.parametrize("kind,pad", [("i8", 0), ("i8", 3), ("i8", 16), ("f16", 0), ("f16", 1), ("f16", 8)])
@pytest.mark.parametrize("tokens,rows,k,n", FEW_DENSE)
def test_dense_products_of_a_few_rows(tokens, rows, k, n, kind, pad):
    check((tokens, 1, 1), rows, k, n, kind, pad, False, 0, True)


@pytest.mark.parametrize("kind,pad", [("i8", 0), ("i8", 3), ("f16", 0), ("f16", 1)])
@pytest.mark.parametrize("tokens,rows,k,n", FEW_GROUPED)
def test_grouped_products_of_a_few_rows(tokens, rows, k, n, kind, pad):
    check((tokens, 1, 1), rows - 3, k, n, kind, pad, True, 0, True)


def test_the_sums_of_all_tiles_are_long_enough_for_several_windows():
    for case in (DENSE, GROUPED):
        assert {t for t, _, k, _ in case if k > 1024} >= {(32, 1, 1), (64, 1, 1), (128, 2, 1), (192, 2, 1)}
    L = H.prepare_linear(weight_codes(2, 130, 5000, 1), scales=torch.ones(2, 130, device="cuda"))
    assert all(int(v) & 2 for v in L.windows.tolist())      # more than 1024 codes of a channel are not exact


def test_ragged_rows_add_up():
    for rows in (30, 197, 297, 697, 997, 1297, 2497, 5997, 6386):
        c = ragged(rows)
        assert len(c) == EXPERTS and sum(c) == rows and min(c) >= 0 and np.count_nonzero(c) >= 5
