"""Refusals of the products with 4-bit weights, on the host: every argument error is returned before any launch."""
import ctypes

import pytest

from paper_2608_01653_gb300 import hatq as H

P = 1 << 30                                         # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return H.load()


def weights(n=64, k=130, group=32, data=P, bias=None):
    return H.Linear4WeightsStruct(n, k, group, 0, data, bias)


def product(lib, L=None, **kw):
    a = dict(x=3 * P, x_type=H.BF16, ldx=130, s_x=None, rows=4)
    b = dict(y_type=H.F16, y=4 * P, ldy=64)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    return lib.hatq_linear4(*a.values(), ctypes.byref(weights() if L is None else L), *b.values(), None)


WEIGHTS = [(dict(n=0), H.ERR_INVALID_ARG), (dict(k=0), H.ERR_INVALID_ARG), (dict(k=(1 << 20) + 1), H.ERR_UNSUPPORTED),
           (dict(n=(1 << 27) + 1), H.ERR_UNSUPPORTED), (dict(group=0), H.ERR_INVALID_ARG), (dict(group=16), H.ERR_INVALID_ARG),
           (dict(group=48), H.ERR_INVALID_ARG), (dict(group=-32), H.ERR_INVALID_ARG)]
BUFFERS = [dict(data=None), dict(data=P + 8), dict(bias=P + 2)]


@pytest.mark.parametrize("kw,status", WEIGHTS + [(b, H.ERR_INVALID_ARG) for b in BUFFERS])
def test_weights_that_are_refused(lib, kw, status):
    assert product(lib, weights(**kw), ldx=1 << 21, ldy=1 << 28) == status and H.last_error()
    assert lib.hatq_linear4_layout(3 * P, 1 << 21, 4 * P, 1 << 21, ctypes.byref(weights(**kw)), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(x_type=3), H.ERR_INVALID_ARG), (dict(y_type=-1), H.ERR_INVALID_ARG), (dict(rows=-1), H.ERR_INVALID_ARG),
    (dict(rows=(1 << 20) + 1), H.ERR_UNSUPPORTED), (dict(ldx=129), H.ERR_INVALID_ARG), (dict(ldy=63), H.ERR_INVALID_ARG),
    (dict(ldx=1 << 33), H.ERR_UNSUPPORTED), (dict(x=None), H.ERR_INVALID_ARG), (dict(y=None), H.ERR_INVALID_ARG),
    (dict(x=3 * P + 1), H.ERR_INVALID_ARG), (dict(y=4 * P + 2, y_type=H.F32), H.ERR_INVALID_ARG), (dict(s_x=P + 2), H.ERR_INVALID_ARG),
    (dict(y=3 * P + 256), H.ERR_INVALID_ARG)])
def test_linear4_refuses(lib, kw, status):
    assert product(lib, **kw) == status and H.last_error()


def test_no_rows_is_no_work(lib):
    assert product(lib, weights(data=None), x=None, y=None, rows=0) == H.OK
    assert lib.hatq_quantize_groups(None, 0, 64, 0, 64, 1, 32, None, 64, None, 2, None) == H.OK
    assert lib.hatq_linear4(3 * P, 0, 130, None, 4, None, 0, 4 * P, 64, None) == H.ERR_INVALID_ARG


def test_sizes(lib):
    a = ctypes.c_size_t()
    for n, k, group, size in ((1, 1, 32, 512 + 128), (17, 65, 64, 2 * 2 * (512 + 64)), (17, 65, 128, 2 * (1024 + 64)),
                              (4096, 4096, 128, 4096 * 2048 + 4096 * 32 * 4), (16, 300, 96, 5 * (512 + 128))):
        assert lib.hatq_linear4_sizes(n, k, group, ctypes.byref(a)) == H.OK and a.value == size
    for kw, status in WEIGHTS:
        L = weights(**kw)
        assert lib.hatq_linear4_sizes(L.n, L.k, L.group, ctypes.byref(a)) == status
    assert lib.hatq_linear4_sizes(1, 1, 32, None) == H.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(w=None), H.ERR_INVALID_ARG), (dict(scales=None), H.ERR_INVALID_ARG), (dict(scales=2 * P + 2), H.ERR_INVALID_ARG),
    (dict(ldw=129), H.ERR_INVALID_ARG), (dict(lds=4), H.ERR_INVALID_ARG), (dict(ldw=1 << 33), H.ERR_UNSUPPORTED)])
def test_layout_refuses(lib, kw, status):
    a = dict(w=3 * P, ldw=130, scales=4 * P, lds=5)
    a.update(kw)
    assert lib.hatq_linear4_layout(*a.values(), ctypes.byref(weights()), None) == status and H.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), H.ERR_INVALID_ARG), (dict(n=-1), H.ERR_INVALID_ARG), (dict(k=0), H.ERR_INVALID_ARG),
    (dict(k=32832, ldw=32832, ldc=32832, lds=1026), H.ERR_UNSUPPORTED), (dict(hb=3), H.ERR_INVALID_ARG), (dict(hb=128), H.ERR_INVALID_ARG),
    (dict(group=8), H.ERR_INVALID_ARG), (dict(ldw=63), H.ERR_INVALID_ARG), (dict(ldc=63), H.ERR_INVALID_ARG),
    (dict(lds=1), H.ERR_INVALID_ARG), (dict(lds=1 << 33), H.ERR_UNSUPPORTED), (dict(w=None), H.ERR_INVALID_ARG),
    (dict(codes=None), H.ERR_INVALID_ARG), (dict(scales=None), H.ERR_INVALID_ARG), (dict(w=P + 1), H.ERR_INVALID_ARG),
    (dict(codes=P + 64), H.ERR_INVALID_ARG), (dict(scales=P + 16), H.ERR_INVALID_ARG), (dict(scales=2 * P + 4), H.ERR_INVALID_ARG)])
def test_quantize_groups_refuses(lib, kw, status):
    a = dict(w=P, type=H.BF16, ldw=64, n=4, k=64, hb=64, group=32, codes=2 * P, ldc=64, scales=3 * P, lds=2)
    a.update(kw)
    assert lib.hatq_quantize_groups(*a.values(), None) == status and H.last_error()


def test_struct_matches_the_header():
    import os
    import subprocess
    import tempfile
    src = ('#include <stdio.h>\n#include <stddef.h>\n#include "hatq.h"\nint main(void) { printf("%zu %zu %zu %zu",'
           ' sizeof(hatq_linear4_weights), offsetof(hatq_linear4_weights, group), offsetof(hatq_linear4_weights, data),'
           ' offsetof(hatq_linear4_weights, bias)); return 0; }\n')
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(src)
        subprocess.run(["gcc", "-I", include, os.path.join(d, "t.c"), "-o", os.path.join(d, "t")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "t")], capture_output=True, text=True).stdout.split()]
    S = H.Linear4WeightsStruct
    assert got == [ctypes.sizeof(S), S.group.offset, S.data.offset, S.bias.offset]
