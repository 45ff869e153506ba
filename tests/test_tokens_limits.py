"""Sizes beyond what the token operators' indices hold are refused on the host, before any launch."""
import ctypes

import pytest

from paper_2608_01653_gb300 import hatq as H

P = 1 << 20                                         # an aligned address that nothing dereferences
MOST_CHANNELS = (1 << 31) - 1024
MOST_VALUES = (1 << 31) - 4096


@pytest.fixture(scope="module")
def lib():
    return H.load()


def weights(n, k=64):
    return H.LinearWeightsStruct(1, n, k, 0, P, P, P, None)


@pytest.mark.parametrize("n", [MOST_CHANNELS + 1, (1 << 31) - 128, (1 << 31) - 1])
def test_more_channels_than_an_index_holds(lib, n):
    size = ctypes.c_size_t(3)
    assert lib.hatq_linear_sizes(1, n, 64, ctypes.byref(size)) == H.ERR_UNSUPPORTED and size.value == 3
    L = weights(n)
    assert lib.hatq_linear_layout(2 * P, 64, ctypes.byref(L), None) == H.ERR_UNSUPPORTED
    assert lib.hatq_linear(2 * P, 0, 64, 3 * P, 4, ctypes.byref(L), 0, 1 << 45, n, None, 0, None) == H.ERR_UNSUPPORTED
    assert lib.hatq_linear_workspace(2 * P, 0, 64, 4, ctypes.byref(L), ctypes.byref(size)) == H.ERR_UNSUPPORTED


def test_as_many_channels_as_an_index_holds(lib):
    size = ctypes.c_size_t()
    assert lib.hatq_linear_sizes(1, MOST_CHANNELS, 65, ctypes.byref(size)) == H.OK and size.value == MOST_CHANNELS * 128


@pytest.mark.parametrize("kind", [H.F32, H.F16, H.BF16])
@pytest.mark.parametrize("c", [MOST_VALUES + 1, (1 << 31) - 1])
def test_combine_rows_wider_than_an_index(lib, kind, c):
    assert lib.hatq_combine_rows(1 << 40, kind, c, 1, P, 2 * P, 1, 1, c, 1 << 45, c, None) == H.ERR_UNSUPPORTED
    assert H.last_error()


def test_linear_plan_refuses(lib):
    plan, L = (ctypes.c_int * 5)(), weights(64)
    ask = lambda x=P, fmt=0, rows=4, L=ctypes.byref(L), out=plan: lib.hatq_linear_plan(x, fmt, 64, rows, L, 0, 0, out)
    assert ask(fmt=2) == ask(rows=0) == ask(rows=-1) == ask(L=None) == ask(out=None) == H.ERR_INVALID_ARG
    assert ask(rows=1 << 31) == H.ERR_UNSUPPORTED
