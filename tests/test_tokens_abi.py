"""Refusals of the token operators, on the host: every argument error is returned before any launch."""
import ctypes

import pytest

from paper_2608_01653_gb300 import hatq as H

P = 1 << 20                                         # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return H.load()


def weights(experts=1, n=64, k=128, codes=P, windows=P, s_w=P, bias=None):
    return H.LinearWeightsStruct(experts, n, k, 0, codes, windows, s_w, bias)


def quantize(lib, **kw):
    a = dict(x=P, x_type=H.BF16, ldx=64, src_rows=4, index=None, rows=4, c=64, hb=64, act=0, gated=0,
             fmt=H.CODES_I8, codes=2 * P, ldc=64, scales=3 * P)
    a.update(kw)
    return lib.hatq_quantize_tokens(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(x_type=3), H.ERR_INVALID_ARG), (dict(x_type=-1), H.ERR_INVALID_ARG), (dict(fmt=2), H.ERR_INVALID_ARG),
    (dict(act=4), H.ERR_INVALID_ARG), (dict(gated=2), H.ERR_INVALID_ARG), (dict(rows=-1), H.ERR_INVALID_ARG),
    (dict(src_rows=-1), H.ERR_INVALID_ARG), (dict(c=0), H.ERR_INVALID_ARG),
    (dict(c=65536, ldx=65536, ldc=65536), H.ERR_UNSUPPORTED), (dict(rows=1 << 31, src_rows=1 << 31), H.ERR_UNSUPPORTED),
    (dict(hb=0), H.ERR_INVALID_ARG), (dict(hb=48), H.ERR_INVALID_ARG), (dict(hb=128), H.ERR_INVALID_ARG),
    (dict(hb=512, c=512, ldx=512, ldc=512), H.ERR_INVALID_ARG), (dict(ldx=63), H.ERR_INVALID_ARG),
    (dict(gated=1), H.ERR_INVALID_ARG), (dict(ldc=63), H.ERR_INVALID_ARG), (dict(ldx=1 << 33), H.ERR_UNSUPPORTED),
    (dict(src_rows=3), H.ERR_INVALID_ARG), (dict(x=None), H.ERR_INVALID_ARG), (dict(codes=None), H.ERR_INVALID_ARG),
    (dict(scales=None), H.ERR_INVALID_ARG), (dict(x=P + 1), H.ERR_INVALID_ARG), (dict(scales=P + 2), H.ERR_INVALID_ARG),
    (dict(index=P + 1), H.ERR_INVALID_ARG), (dict(codes=2 * P + 1, fmt=H.CODES_F16), H.ERR_INVALID_ARG),
    (dict(codes=P + 256), H.ERR_INVALID_ARG)])
def test_quantize_tokens_refuses(lib, kw, status):
    assert quantize(lib, **kw) == status
    assert H.last_error()


def test_no_rows_is_no_work(lib):
    assert quantize(lib, rows=0, src_rows=0, x=None, codes=None, scales=None) == H.OK
    L = weights()
    assert lib.hatq_linear(None, 0, 128, None, 0, ctypes.byref(L), 0, None, 64, None, 0, None) == H.OK
    assert lib.hatq_grouped_linear(None, 0, 128, None, 0, None, ctypes.byref(L), 0, None, 64, None, 0, None) == H.OK
    assert lib.hatq_combine_rows(None, 0, 8, 0, None, None, 0, 1, 8, None, 8, None) == H.OK


def test_linear_sizes(lib):
    size = ctypes.c_size_t()
    for e, n, k, want in ((1, 1, 1, 128 * 64), (3, 129, 65, 3 * 256 * 128), (64, 4096, 65536, 64 * 4096 * 65536)):
        assert lib.hatq_linear_sizes(e, n, k, ctypes.byref(size)) == H.OK and size.value == want
    for e, n, k, st in ((0, 1, 1, H.ERR_INVALID_ARG), (1025, 1, 1, H.ERR_INVALID_ARG), (1, 0, 1, H.ERR_INVALID_ARG),
                        (1, 1, 0, H.ERR_INVALID_ARG), (1, 1, 65537, H.ERR_UNSUPPORTED)):
        assert lib.hatq_linear_sizes(e, n, k, ctypes.byref(size)) == st
    assert lib.hatq_linear_sizes(1, 1, 1, None) == H.ERR_INVALID_ARG


def product(lib, L=None, **kw):
    a = dict(x=2 * P, fmt=H.CODES_F16, ldx=128, s_x=3 * P, rows=40, y_type=H.BF16, y=4 * P, ldy=64, ws=None, size=0)
    a.update(kw)
    L = L if L is not None else weights()
    return lib.hatq_linear(a["x"], a["fmt"], a["ldx"], a["s_x"], a["rows"], ctypes.byref(L), a["y_type"], a["y"],
                           a["ldy"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(fmt=2), H.ERR_INVALID_ARG), (dict(y_type=5), H.ERR_INVALID_ARG), (dict(rows=-1), H.ERR_INVALID_ARG),
    (dict(rows=1 << 31), H.ERR_UNSUPPORTED), (dict(ldx=127), H.ERR_INVALID_ARG), (dict(ldy=63), H.ERR_INVALID_ARG),
    (dict(ldy=1 << 33), H.ERR_UNSUPPORTED), (dict(x=None), H.ERR_INVALID_ARG), (dict(s_x=None), H.ERR_INVALID_ARG),
    (dict(y=None), H.ERR_INVALID_ARG), (dict(x=2 * P + 1), H.ERR_INVALID_ARG), (dict(y=4 * P + 1), H.ERR_INVALID_ARG),
    (dict(s_x=3 * P + 2), H.ERR_INVALID_ARG), (dict(y=2 * P + 64), H.ERR_INVALID_ARG),
    (dict(L=weights(codes=None)), H.ERR_INVALID_ARG), (dict(L=weights(codes=P + 8)), H.ERR_INVALID_ARG),
    (dict(L=weights(windows=None)), H.ERR_INVALID_ARG), (dict(L=weights(s_w=None)), H.ERR_INVALID_ARG),
    (dict(L=weights(bias=P + 2)), H.ERR_INVALID_ARG), (dict(L=weights(experts=2)), H.ERR_INVALID_ARG),
    (dict(L=weights(experts=0)), H.ERR_INVALID_ARG), (dict(L=weights(n=0)), H.ERR_INVALID_ARG),
    (dict(L=weights(k=65537), ldx=65537), H.ERR_UNSUPPORTED)])
def test_linear_refuses(lib, kw, status):
    assert product(lib, **kw) == status
    assert H.last_error()


def test_grouped_linear_refuses(lib):
    L = weights(experts=4)
    call = lambda rows, off, y: lib.hatq_grouped_linear(2 * P, H.CODES_F16, 128, 3 * P, rows, off, ctypes.byref(L), H.F32, y, 64,
                                                        None, 0, None)
    assert call(40, None, 4 * P) == H.ERR_INVALID_ARG
    assert call(40, P + 1, 4 * P) == H.ERR_INVALID_ARG
    assert call(40, 5 * P, 2 * P) == H.ERR_INVALID_ARG
    assert lib.hatq_grouped_linear(2 * P, 0, 128, 3 * P, 4, 5 * P, None, 0, 4 * P, 64, None, 0, None) == H.ERR_INVALID_ARG


def test_layout_refuses(lib):
    L = weights()
    assert lib.hatq_linear_layout(None, 128, ctypes.byref(L), None) == H.ERR_INVALID_ARG
    assert lib.hatq_linear_layout(2 * P, 127, ctypes.byref(L), None) == H.ERR_INVALID_ARG
    assert lib.hatq_linear_layout(2 * P, 128, None, None) == H.ERR_INVALID_ARG
    assert lib.hatq_linear_layout(2 * P, 128, ctypes.byref(weights(codes=P + 4)), None) == H.ERR_INVALID_ARG
    assert lib.hatq_linear_layout(2 * P, 1 << 33, ctypes.byref(L), None) == H.ERR_UNSUPPORTED


def test_workspace(lib):
    size = ctypes.c_size_t(7)
    L = weights(k=130)
    ask = lambda x, fmt, ldx, rows: (lib.hatq_linear_workspace(x, fmt, ldx, rows, ctypes.byref(L), ctypes.byref(size)), size.value)
    assert ask(P, H.CODES_F16, 136, 1000) == (H.OK, 0)                  # goes to the tensor cores as it lies
    assert ask(P, H.CODES_I8, 144, 0) == (H.OK, 0)
    assert ask(P, H.CODES_I8, 144, 1) == (H.OK, 0)                      # the dot-product kernel takes any codes
    for x, fmt, ldx in ((P, H.CODES_I8, 144), (P, H.CODES_F16, 131), (P + 2, H.CODES_F16, 136)):
        assert ask(x, fmt, ldx, 1000) == (H.OK, 1000 * 192 * 2)
    assert ask(P, 9, 144, 1)[0] == H.ERR_INVALID_ARG
    assert ask(P, 0, 144, -1)[0] == H.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), H.ERR_INVALID_ARG), (dict(rows=-1), H.ERR_INVALID_ARG), (dict(tokens=-1), H.ERR_INVALID_ARG),
    (dict(c=0), H.ERR_INVALID_ARG), (dict(topk=0), H.ERR_INVALID_ARG), (dict(topk=65), H.ERR_INVALID_ARG),
    (dict(rows=1 << 31), H.ERR_UNSUPPORTED), (dict(ldy=7), H.ERR_INVALID_ARG), (dict(ldo=7), H.ERR_INVALID_ARG),
    (dict(ldy=1 << 33), H.ERR_UNSUPPORTED), (dict(y=None), H.ERR_INVALID_ARG), (dict(index=None), H.ERR_INVALID_ARG),
    (dict(weights=None), H.ERR_INVALID_ARG), (dict(out=None), H.ERR_INVALID_ARG), (dict(y=P + 1), H.ERR_INVALID_ARG),
    (dict(out=P), H.ERR_INVALID_ARG)])
def test_combine_rows_refuses(lib, kw, status):
    a = dict(y=P, type=H.F16, ldy=8, rows=16, index=2 * P, weights=3 * P, tokens=4, topk=2, c=8, out=4 * P, ldo=8)
    a.update(kw)
    assert lib.hatq_combine_rows(*a.values(), None) == status
    assert H.last_error()


def test_struct_matches_the_header():
    import os
    import subprocess
    import tempfile
    src = ('#include <stdio.h>\n#include <stddef.h>\n#include "hatq.h"\nint main(void) { printf("%zu %zu %zu %zu %zu",'
           ' sizeof(hatq_linear_weights), offsetof(hatq_linear_weights, codes), offsetof(hatq_linear_weights, windows),'
           ' offsetof(hatq_linear_weights, s_w), offsetof(hatq_linear_weights, bias)); return 0; }\n')
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(src)
        subprocess.run(["gcc", "-I", include, os.path.join(d, "t.c"), "-o", os.path.join(d, "t")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "t")], capture_output=True, text=True).stdout.split()]
    S = H.LinearWeightsStruct
    assert got == [ctypes.sizeof(S), S.codes.offset, S.windows.offset, S.s_w.offset, S.bias.offset]
