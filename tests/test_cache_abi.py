"""Refusals of the 4-bit cache's operators, on the host: every argument error is returned before any launch."""
import ctypes

import pytest

from paper_2608_01653_gb300 import hatq as H

P = 1 << 30                                         # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return H.load()


def cache(data=P, pages=4, page=64, heads=2, width=128, hb=128):
    return H.TokenCacheStruct(data, pages, page, heads, width, hb, 0)


def append(lib, c=None, **kw):
    a = dict(k=2 * P, ldk=256, hk=128, v=3 * P, ldv=256, hv=128, type=H.BF16, rows=4, table=4 * P, ldt=3, width=3,
             lengths=5 * P, starts=6 * P, seqs=2, kept_k=7 * P, kept_v=8 * P)
    a.update(kw)
    c = cache() if c is None else c
    return lib.hatq_append_tokens(ctypes.byref(c), *a.values(), None)


CACHES = [(dict(width=96), H.ERR_UNSUPPORTED), (dict(width=0), H.ERR_UNSUPPORTED), (dict(page=8), H.ERR_UNSUPPORTED),
          (dict(page=128), H.ERR_UNSUPPORTED), (dict(heads=0), H.ERR_INVALID_ARG), (dict(heads=1025), H.ERR_INVALID_ARG),
          (dict(pages=-1), H.ERR_INVALID_ARG), (dict(hb=0), H.ERR_INVALID_ARG), (dict(hb=48), H.ERR_INVALID_ARG),
          (dict(hb=256), H.ERR_INVALID_ARG), (dict(width=192, hb=128), H.ERR_INVALID_ARG), (dict(data=None), H.ERR_INVALID_ARG),
          (dict(data=P + 8), H.ERR_INVALID_ARG)]
SEQUENCES = [(dict(rows=-1), H.ERR_INVALID_ARG), (dict(seqs=-1), H.ERR_INVALID_ARG), (dict(width=-1), H.ERR_INVALID_ARG),
             (dict(seqs=65537), H.ERR_UNSUPPORTED), (dict(rows=1 << 31), H.ERR_UNSUPPORTED),
             (dict(starts=None), H.ERR_INVALID_ARG), (dict(width=(1 << 24) + 1), H.ERR_UNSUPPORTED),
             (dict(ldt=-1), H.ERR_INVALID_ARG), (dict(lengths=None), H.ERR_INVALID_ARG), (dict(table=None), H.ERR_INVALID_ARG),
             (dict(table=4 * P + 2), H.ERR_INVALID_ARG), (dict(lengths=5 * P + 1), H.ERR_INVALID_ARG),
             (dict(starts=6 * P + 2), H.ERR_INVALID_ARG)]


@pytest.mark.parametrize("kw,status", CACHES)
def test_caches_that_are_refused(lib, kw, status):
    assert append(lib, cache(**kw)) == status and H.last_error()
    assert attend(lib, cache(**kw)) == status and H.last_error()
    size = ctypes.c_size_t(7)
    assert lib.hatq_attend_workspace(ctypes.byref(cache(**kw)), H.BF16, 4, 4, 2, 1, 3, ctypes.byref(size)) == status
    assert size.value == 7


@pytest.mark.parametrize("kw,status", SEQUENCES + [
    (dict(type=3), H.ERR_INVALID_ARG), (dict(k=None), H.ERR_INVALID_ARG), (dict(v=None), H.ERR_INVALID_ARG),
    (dict(k=2 * P + 1), H.ERR_INVALID_ARG), (dict(v=3 * P + 2, type=H.F32), H.ERR_INVALID_ARG),
    (dict(ldk=-1), H.ERR_INVALID_ARG), (dict(hv=-128), H.ERR_INVALID_ARG), (dict(ldv=1 << 33), H.ERR_UNSUPPORTED),
    (dict(kept_k=None), H.ERR_INVALID_ARG), (dict(kept_v=None), H.ERR_INVALID_ARG), (dict(kept_k=7 * P + 8), H.ERR_INVALID_ARG),
    (dict(kept_k=8 * P), H.ERR_INVALID_ARG), (dict(kept_v=2 * P + 256), H.ERR_INVALID_ARG), (dict(kept_k=P), H.ERR_INVALID_ARG),
    (dict(k=P + 512), H.ERR_INVALID_ARG), (dict(rows=1 << 30, seqs=4), H.ERR_UNSUPPORTED)])
def test_append_refuses(lib, kw, status):
    assert append(lib, **kw) == status and H.last_error()


@pytest.mark.parametrize("kw", [dict(k=P + 512, ldk=0), dict(v=P + 512, ldv=0), dict(k=P + 512, ldk=0, ldv=0)])
def test_append_refuses_one_row_for_all_within_the_cache(lib, kw):
    """Keys or values expanded over the rows (a pitch of 0) that lie in a cache of one page."""
    assert append(lib, cache(pages=1), **kw) == H.ERR_INVALID_ARG and "overlap" in H.last_error()
    assert append(lib, cache(pages=1), **dict(kw, rows=1, seqs=1)) == H.ERR_INVALID_ARG


def attend(lib, c=None, **kw):
    a = dict(q=2 * P, type=H.BF16, ldq=512, hq=128, heads=4, rows=4, table=4 * P, ldt=3, width=3, lengths=5 * P, starts=6 * P,
             seqs=2, scale=0.1, out=7 * P, ldo=512, ho=128, ws=8 * P, size=1 << 40)
    a.update(kw)
    a = list(a.values())
    c = cache() if c is None else c
    return lib.hatq_attend_tokens(*a[:6], ctypes.byref(c), *a[6:], None)


@pytest.mark.parametrize("kw,status", SEQUENCES + [
    (dict(type=H.F32), H.ERR_INVALID_ARG), (dict(heads=0), H.ERR_INVALID_ARG), (dict(heads=3), H.ERR_INVALID_ARG),
    (dict(heads=32768), H.ERR_UNSUPPORTED), (dict(rows=1 << 30, seqs=4), H.ERR_UNSUPPORTED),
    (dict(scale=float("inf")), H.ERR_INVALID_ARG), (dict(scale=float("nan")), H.ERR_INVALID_ARG),
    (dict(q=None), H.ERR_INVALID_ARG), (dict(out=None), H.ERR_INVALID_ARG), (dict(q=2 * P + 1), H.ERR_INVALID_ARG),
    (dict(ldo=511), H.ERR_INVALID_ARG), (dict(ho=127), H.ERR_INVALID_ARG), (dict(ldo=0), H.ERR_INVALID_ARG),
    (dict(hq=-1), H.ERR_INVALID_ARG), (dict(ldq=1 << 33), H.ERR_UNSUPPORTED), (dict(out=2 * P + 1024), H.ERR_INVALID_ARG),
    (dict(out=P + 64), H.ERR_INVALID_ARG), (dict(out=2 * P, ldo=128, ho=512), H.ERR_INVALID_ARG)])
def test_attend_refuses(lib, kw, status):
    assert attend(lib, **kw) == status and H.last_error()


@pytest.mark.parametrize("scale", [2.5e38, -3.4e38])                    # times log2(e): above the largest fp32
def test_attend_refuses_scales_that_overflow(lib, scale):
    assert attend(lib, scale=scale) == H.ERR_INVALID_ARG and b"finite" in H.last_error().encode()


def test_no_rows_is_no_work(lib):
    none = dict(rows=0, seqs=0, table=None, lengths=None, starts=None)
    assert append(lib, k=None, v=None, kept_k=None, kept_v=None, **none) == H.OK
    assert append(lib, cache(data=None, pages=0), k=None, v=None, **none) == H.OK
    assert append(lib, seqs=0, lengths=None) == H.OK                    # rows of no sequence
    assert attend(lib, q=None, out=None, ws=None, size=0, **none) == H.OK
    size = ctypes.c_size_t(7)
    assert lib.hatq_attend_workspace(ctypes.byref(cache()), H.BF16, 4, 0, 0, 0, 3, ctypes.byref(size)) == H.OK and size.value == 0


def test_struct_matches_the_header():
    import os
    import subprocess
    import tempfile
    src = ('#include <stdio.h>\n#include <stddef.h>\n#include "hatq.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu",'
           ' sizeof(hatq_token_cache), offsetof(hatq_token_cache, pages), offsetof(hatq_token_cache, page),'
           ' offsetof(hatq_token_cache, heads), offsetof(hatq_token_cache, width), offsetof(hatq_token_cache, hb)); return 0; }\n')
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(src)
        subprocess.run(["gcc", "-I", include, os.path.join(d, "t.c"), "-o", os.path.join(d, "t")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "t")], capture_output=True, text=True).stdout.split()]
    S = H.TokenCacheStruct
    assert got == [ctypes.sizeof(S), S.pages.offset, S.page.offset, S.heads.offset, S.width.offset, S.hb.offset]
