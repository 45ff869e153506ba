"""The 4-bit cache on the GPU against plain formulas.

What append stores is compared exactly, with the formula in single precision on
the host. What attend returns is compared with the formula in 64 bits; its bound
is eight standard deviations of the kernel's roundings (see `reference`) and
half a step of the output type.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INF, NAN = math.inf, math.nan


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def finish():
    torch.cuda.synchronize()
    H.sync_status()


class Run:
    """Sequences in a cache of random bytes: lengths and new tokens of each, pages in no order, a table that is wider
    than need be and says -1 behind a sequence's pages."""

    def __init__(self, lengths, new, kv=2, width=128, page=64, hb=None, dtype="bf16", seed=1, spare=2, one_each=False):
        self.kv, self.width, self.page, self.hb = kv, width, page, (width & -width) if hb is None else hb
        self.dtype, self.new, self.len = TYPES[dtype], new, lengths
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + spare
        order = torch.randperm(pages, generator=gen(seed), device="cuda").tolist()
        rows, at = [], 0
        for u in used:
            rows.append(order[at:at + u] + [-1] * (max(used) + 1 - u))
            at += u
        self.table = torch.tensor(rows, dtype=torch.int32, device="cuda").reshape(len(lengths), -1)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.starts = None if one_each else torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        self.rows = sum(new)
        data = torch.randint(0, 256, (pages, kv, page * (width + 8)), generator=gen(seed + 1), device="cuda").to(torch.uint8)
        scales = 0.3 * torch.exp(0.5 * torch.randn(pages, kv, 2 * page, generator=gen(seed + 2), device="cuda"))
        data[:, :, page * width:] = scales.view(torch.uint8)
        self.cache = H.TokenCache(data, page, self.hb)

    def random(self, heads, seed, rows=None):
        return torch.randn(rows or self.rows, heads, self.width, generator=gen(seed), device="cuda").to(self.dtype)

    def places(self):
        """(row, sequence, position) of every new token."""
        r = 0
        for b, (n, m) in enumerate(zip(self.len, self.new)):
            for i in range(m):
                yield r, b, n - m + i
                r += 1


# ------------------------------------------------------------------ append

def quantized(x, hb):
    """Codes, scales and kept values of [rows][heads][width] in single precision, as the header states them."""
    t, h = x.float().cpu().numpy(), 1
    shape = t.shape
    with np.errstate(all="ignore"):
        while h < hb:
            t = t.reshape(*shape[:-1], -1, 2, h)
            t = np.stack([t[..., 0, :] + t[..., 1, :], t[..., 0, :] - t[..., 1, :]], -2).reshape(shape)
            h *= 2
        a = np.abs(t).max(-1, keepdims=True)                            # (NaN stays)
        sound = np.isfinite(np.float32(7) * a)
        live = sound & (a > 0)
        codes = np.where(live, np.rint(np.float32(7) * t / np.where(live, a, 1)), 0).astype(np.float32)
        inv = np.float32(1 / math.sqrt(hb))
        scale = np.where(sound, np.where(live, a / np.float32(7), np.float32(1)) * inv, np.float32(NAN)).astype(np.float32)
        back, h = codes, 1
        while h < hb:
            back = back.reshape(*shape[:-1], -1, 2, h)
            back = np.stack([back[..., 0, :] + back[..., 1, :], back[..., 0, :] - back[..., 1, :]], -2).reshape(shape)
            h *= 2
        kept = torch.from_numpy(back * (scale * inv)).to(x.dtype)
    return codes.astype(np.int64), scale[..., 0], kept


def appended(run, k, v):
    """The cache's bytes after an append, and the kept values."""
    data = run.cache.data.cpu().numpy().copy()
    half, page, width = run.width // 2, run.page, run.width
    table = run.table.cpu().numpy()
    kept = []
    for part, x in enumerate((k, v)):
        codes, scale, back = quantized(x, run.hb)
        kept.append(back)
        for r, b, at in run.places():
            if at < 0:
                continue
            p = table[b, at // page]
            if not 0 <= p < data.shape[0]:
                continue
            n = (codes[r] + 8).astype(np.uint8)
            i = part * page + at % page
            data[p, :, i * half:(i + 1) * half] = n[:, 0::2] | n[:, 1::2] << 4
            data[p, :, page * width + 4 * i:page * width + 4 * i + 4] = scale[r][:, None].view(np.uint8)
    return torch.from_numpy(data), kept


def same(a, b):
    """Bit for bit; NaNs count as equal."""
    a, b = a.cpu(), b.cpu()
    return torch.equal(a.nan_to_num(nan=12345.0), b.nan_to_num(nan=12345.0)) and torch.equal(a.isnan(), b.isnan())


def check_append(run, k, v, kept=True):
    want, back = appended(run, k, v)
    got = H.append_tokens(run.cache, k, v, run.table, run.lengths, run.starts, kept=kept)
    finish()
    size = run.page * run.width
    assert torch.equal(run.cache.data[:, :, :size].cpu(), want[:, :, :size])
    assert same(run.cache.data[:, :, size:].contiguous().view(torch.float32), want[:, :, size:].contiguous().view(torch.float32))
    if kept:
        n = sum(run.new)
        assert same(got[0][:n], back[0][:n]) and same(got[1][:n], back[1][:n])
    else:
        assert got is None


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("width,hb", [(64, 1), (64, 2), (64, 64), (128, 4), (128, 32), (128, 128), (192, 8), (192, 64), (256, 16),
                                      (256, 256)])
@pytest.mark.parametrize("page", [16, 64])
def test_append_stores_the_formulas_codes(dtype, width, hb, page):
    run = Run([130, 1, 64, 17], [130, 1, 3, 17], kv=3, width=width, page=page, hb=hb, dtype=dtype)
    check_append(run, run.random(3, 5), run.random(3, 6))


@pytest.mark.parametrize("seqs", [1, 2, 33, 70])
def test_append_one_token_each(seqs):
    run = Run([1 + 7 * i for i in range(seqs)], [1] * seqs, kv=5, width=128, page=32, one_each=True)
    check_append(run, run.random(5, 5), run.random(5, 6), kept=False)


def test_append_sequences_without_tokens_and_rows_without_sequences():
    run = Run([0, 5, 40, 0, 3], [0, 2, 40, 0, 3], kv=1, width=64, page=16)
    k, v = run.random(1, 5, run.rows + 4), run.random(1, 6, run.rows + 4)
    check_append(run, k, v)
    before = run.cache.data.clone()
    H.append_tokens(run.cache, k, v, run.table, run.lengths, torch.zeros_like(run.starts))
    finish()
    assert torch.equal(run.cache.data, before)


def test_append_more_rows_than_tokens_and_pages_that_are_none():
    run = Run([3, 70, 40], [8, 70, 40], kv=2, width=64, page=16)
    run.table[1, 1], run.table[1, 2], run.table[2, 0] = -1, 1 << 30, run.cache.pages
    check_append(run, run.random(2, 5), run.random(2, 6))


def test_append_lengths_beyond_the_table():
    """A length is clamped to the table's pages: the last row is its last token."""
    run = Run([32], [4], kv=1, width=64, page=16)
    table = run.table[:, :2]
    k, v = run.random(1, 5), run.random(1, 6)
    want, _ = appended(run, k, v)
    H.append_tokens(run.cache, k, v, table, torch.full_like(run.lengths, 2 ** 31 - 1), run.starts)
    finish()
    assert torch.equal(run.cache.data.cpu(), want)


def test_append_strides():
    """Keys and values as columns of one buffer, then with heads outside rows, then expanded over heads, then unaligned."""
    run = Run([50, 9], [50, 9], kv=4, width=128, page=32)
    both = torch.randn(run.rows, 2, 4, 128, generator=gen(5), device="cuda").bfloat16()
    check_append(run, both[:, 0], both[:, 1])
    out = torch.randn(4, run.rows, 128, generator=gen(6), device="cuda").bfloat16().transpose(0, 1)
    check_append(run, out, both[:, 1])
    check_append(run, both[:, :1, 0].expand(-1, 4, -1), both[:1, 1].expand(run.rows, -1, -1))
    odd = torch.randn(run.rows, 4, 131, generator=gen(7), device="cuda").bfloat16()
    check_append(run, odd[:, :, 3:], odd[:, :, 1:129])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_append_values_at_the_borders(dtype):
    """Zeros, single values, ties between codes, infinities, NaN, the largest and the smallest values of the type."""
    run = Run([16], [16], kv=1, width=64, page=16, hb=1, dtype=dtype)
    info = torch.finfo(run.dtype)
    k, v = run.random(1, 5), torch.zeros(16, 1, 64, dtype=run.dtype, device="cuda")
    k[0, 0] = 0
    k[1, 0], k[1, 0, 7] = 0, -3
    k[2, 0] = torch.arange(64, device="cuda").sub(32).to(run.dtype) / 4.5     # thirds and halves of a code
    k[3, 0] = torch.arange(64, device="cuda").remainder(15).sub(7).to(run.dtype) + 0.5
    k[3, 0, 0] = 7
    k[4, 0, 5], k[5, 0, 6], k[6, 0, 63] = INF, -INF, NAN
    k[7, 0] = info.max
    k[8, 0], k[8, 0, 1] = info.tiny, -info.tiny / 4
    k[9, 0], k[9, 0, 2] = 0, info.smallest_normal * info.eps
    k[10, 0, ::2], k[10, 0, 3] = NAN, INF
    v[:, 0] = k[:, 0].flip(0)
    check_append(run, k, v)


def test_append_into_pages_beyond_4_gb():
    pages = 600_000
    cache = H.TokenCache.empty(pages, 1, 128, page=64, hb=128)               # 5.2 GB
    k, v = (torch.randn(2, 1, 128, generator=gen(s), device="cuda").bfloat16() for s in (5, 6))
    table = torch.tensor([[pages - 1], [3]], dtype=torch.int32, device="cuda")
    H.append_tokens(cache, k, v, table, torch.tensor([64, 64], dtype=torch.int32, device="cuda"))
    finish()
    for part, x in enumerate((k, v)):
        codes, scale, _ = quantized(x, 128)
        for i, p in enumerate((pages - 1, 3)):
            n = (codes[i, 0] + 8).astype(np.uint8)
            at = part * 64 + 63
            assert torch.equal(cache.data[p, 0, at * 64:at * 64 + 64].cpu(), torch.from_numpy(n[0::2] | n[1::2] << 4))
            assert cache.data[p, 0, 64 * 128 + 4 * at:64 * 128 + 4 * at + 4].clone().view(torch.float32).item() == scale[i, 0]


# ------------------------------------------------------------------ attend

def held(run, b, length):
    """Keys and values of a sequence in the transformed basis in 64 bits [kv][length][width], their scales
    [kv][length], and which of its tokens lie in a page."""
    page, width = run.page, run.width
    data = run.cache.data.cpu()
    entries = run.table[b].cpu().tolist()[:-(-length // page)]
    there = torch.tensor([0 <= e < data.shape[0] for e in entries], dtype=torch.bool).repeat_interleave(page)[:length]
    rec = data[[e if 0 <= e < data.shape[0] else 0 for e in entries]]
    n = rec[:, :, :page * width].reshape(len(entries), run.kv, 2, page, width // 2)
    codes = torch.stack([n & 15, n >> 4], -1).double().flatten(-2) - 8
    scales = rec[:, :, page * width:].contiguous().view(torch.float32).reshape(len(entries), run.kv, 2, page).double()
    both = [(codes[:, :, i].transpose(0, 1).reshape(run.kv, -1, width)[:, :length],
             scales[:, :, i].transpose(0, 1).reshape(run.kv, -1)[:, :length]) for i in (0, 1)]
    return *both[0], *both[1], there


def basis(hb):
    i = torch.arange(hb)
    parity = sum(((i[:, None] & i[None]) >> j) & 1 for j in range(8)) % 2
    return (1.0 - 2.0 * parity).double() / math.sqrt(hb)


def turned(x, hb):
    return (x.reshape(*x.shape[:-1], -1, hb) @ basis(hb)).reshape(x.shape)


def reference(run, q, scale=None, rows=None):
    """Outputs in 64 bits and the standard deviation of the kernel's roundings (rows: of some rows only, zeros elsewhere).

    Every rounding is an independent error of zero mean, at most half a step, so of a standard deviation of at most
    h / sqrt(3), h = 2^-11 (bf16: q and w v once to fp16) or 2^-21 (fp16: twice). With n keys and width D:
      s_j    q's roundings h k_jd q_d per product, D / 8 accumulations of 2^-23 of a partial sum (below 15 k sum |q|),
             and 2^-22 of |s| in fp32 products and the exponential's argument; w_j inherits them as relative errors,
             and 2^-21 of its own (exponential)
      o_d    w_j v_jd - o_d times w_j's relative error and h, n / 16 + 64 accumulations of 2^-23 of a partial sum
             (below 15 sum w v), twice, as codes + 8 and 8 are summed apart
    and all of it goes through the transform back, which adds variances / hb within a block."""
    h = (2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21) / math.sqrt(3)
    group, D = q.shape[1] // run.kv, run.width
    scale = D ** -0.5 if scale is None else scale
    out, sd = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    t = turned(q.double().cpu(), run.hb).reshape(q.shape[0], run.kv, group, D)
    got, r = {}, 0
    for b, (n, m) in enumerate(zip(run.len, run.new)):
        kc, ks, vc, vs, there = held(run, b, n) if n else (None,) * 5
        for i in range(m):
            p = n - m + i
            if p >= 0 and (rows is None or r in rows) and bool(there[:p + 1].any()):
                keep = torch.nonzero(there[:p + 1])[:, 0]
                K, V, sv = kc[:, keep] * ks[:, keep, None], vc[:, keep] * vs[:, keep, None], vs[:, keep]
                s = scale * torch.einsum("hgd,hnd->hgn", t[r], K)
                var = (scale * h) ** 2 * torch.einsum("hgd,hnd->hgn", t[r] ** 2, K ** 2)
                var += D / 8 * (scale * 2.0 ** -23 * 15 * t[r].abs().sum(-1)[..., None] * ks[:, None, keep]) ** 2
                var += (2.0 ** -22 * s.abs()) ** 2 + 2.0 ** -42 + h ** 2
                w = torch.softmax(s, -1)
                o = torch.einsum("hgn,hnd->hgd", w, V)
                ov = torch.einsum("hgn,hnd->hgd", w ** 2 * var, V ** 2) + o ** 2 * (w ** 2 * var).sum(-1, keepdim=True)
                ov += 2 * (len(keep) / 16 + 64) * (2.0 ** -23 * 15 * torch.einsum("hgn,hn->hg", w, sv)[..., None]) ** 2
                out[r] = turned(o, run.hb).reshape(q.shape[1:])
                mean = ov.reshape(*ov.shape[:-1], -1, run.hb).mean(-1, keepdim=True).expand(-1, -1, -1, run.hb)
                sd[r] = mean.reshape(q.shape[1:]).sqrt()
            r += 1
    return out, sd


def check_attend(run, q, y, scale=None, rows=None, more=1.0):
    """rows: of these only; more: times the deviation."""
    ref, sd = reference(run, q, scale, rows)
    of = list(range(sum(run.new))) if rows is None else sorted(rows)
    err = (y.double().cpu() - ref)[of].abs()
    tol = (8 * more * sd + torch.finfo(q.dtype).eps / 2 * 1.01 * ref.abs() + 2.0 ** -24)[of]
    assert y.dtype == q.dtype
    worst = float((err / tol).nan_to_num(nan=INF).max())
    assert worst <= 1


def attend(run, q, **kw):
    y = H.attend_tokens(q, run.cache, run.table, run.lengths, run.starts, **kw)
    finish()
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width,hb,page", [(64, 64, 16), (64, 1, 64), (128, 128, 64), (128, 16, 32), (192, 64, 16), (256, 256, 64),
                                           (256, 8, 32)])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_attend_one_token_each(dtype, width, hb, page, group):
    lengths = [1, 2, 15, 16, 63, 64, 65, 129, 700, 0, 1500]
    run = Run(lengths, [1] * len(lengths), kv=2, width=width, page=page, hb=hb, dtype=dtype, one_each=True)
    q = run.random(2 * group, 5)
    check_attend(run, q, attend(run, q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width,page", [(64, 16), (128, 64), (192, 32), (256, 64)])
@pytest.mark.parametrize("kv,group", [(1, 1), (3, 2), (2, 5), (1, 16)])
def test_attend_several_tokens_each(dtype, width, page, kv, group):
    run = Run([1, 40, 130, 64, 0, 5, 260], [1, 3, 130, 17, 0, 9, 1], kv=kv, width=width, page=page, dtype=dtype)
    q = run.random(kv * group, 5)
    check_attend(run, q, attend(run, q))


@pytest.mark.parametrize("heads,kv", [(64, 1), (24, 24)])
def test_attend_many_heads(heads, kv):
    run = Run([300, 77], [1, 1], kv=kv, width=64, one_each=True)
    q = run.random(heads, 5)
    check_attend(run, q, attend(run, q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_a_long_sequence(dtype):
    run = Run([40_000], [2], kv=1, width=128, dtype=dtype)
    q = run.random(4, 5)
    check_attend(run, q, attend(run, q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width", [64, 128, 256])
def test_attend_a_prompt(dtype, width):
    """Every row sees its own prefix, down to a single token."""
    run = Run([513, 100], [513, 37], kv=1, width=width, dtype=dtype)
    q = run.random(2, 5)
    check_attend(run, q, attend(run, q))


@pytest.mark.parametrize("scale", [0.0, 1e-3, 0.7, -0.3, 8.0])
def test_attend_scales(scale):
    """From equal weights to a single key's."""
    run = Run([200, 333], [3, 1], kv=2, width=64)
    q = run.random(4, 5)
    check_attend(run, q, attend(run, q, scale=scale), scale)


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e4, 1e30])
def test_attend_value_scales_of_any_size(size):
    run = Run([200, 333], [3, 1], kv=2, width=64)
    at = run.page * run.width + 4 * run.page
    scales = run.cache.data[:, :, at:].contiguous().view(torch.float32) * size
    run.cache.data[:, :, at:] = scales.view(torch.uint8)
    q = run.random(4, 5)
    y = attend(run, q)
    ref, sd = reference(run, q)
    assert bool(((y.double().cpu() - ref).abs() <= 8 * sd + 2.0 ** -8 * 1.01 * ref.abs() + 2.0 ** -130).all())


def test_attend_queries_of_any_size():
    run = Run([200, 333], [3, 1], kv=2, width=64)
    q = run.random(4, 5) * torch.tensor([1e-30, 1e-6, 1.0, 100.0], device="cuda").bfloat16()[:, None, None]
    check_attend(run, q, attend(run, q))


def test_attend_rows_that_see_nothing():
    """More new tokens than tokens, sequences without tokens, pages that are none: zeros, and no other row changes."""
    run = Run([3, 150, 40, 0, 70], [8, 5, 3, 2, 1], kv=2, width=64, page=16)
    run.table[2, :] = -1
    run.table[1, 3], run.table[1, 5], run.table[4, 4] = -1, 1 << 30, run.cache.pages
    q = run.random(6, 5)
    y = attend(run, q)
    check_attend(run, q, y)
    assert bool((y[:5] == 0).all()) and bool((y[13:18] == 0).all()) and bool((y[5:13] != 0).any())


def test_attend_rows_of_no_sequence_are_left():
    run = Run([40, 9], [3, 2], kv=2, width=64)
    q = run.random(4, 5, 9)
    y = torch.full_like(q, 7.0)
    starts = run.starts + 2                                              # rows 0, 1, 7 and 8 are nobody's
    H.attend_tokens(q, run.cache, run.table, run.lengths, starts, out=y)
    finish()
    assert bool((y[:2] == 7).all()) and bool((y[7:] == 7).all())
    check_attend(run, q[2:7].contiguous(), y[2:7])


def test_attend_offsets_out_of_order_and_range():
    """Offsets that step back count as the largest before them, those behind the rows as the last."""
    run = Run([40, 9, 30, 20], [3, 0, 2, 4], kv=2, width=64)
    q = run.random(4, 5)
    y = H.attend_tokens(q, run.cache, run.table, run.lengths, torch.tensor([-5, 3, 1, 5, 1 << 30], dtype=torch.int32, device="cuda"))
    finish()
    check_attend(run, q, y)


def test_attend_what_a_row_does_not_see():
    """NaN and infinite scales behind a row's position, behind the last token, in other pages: no trace."""
    run = Run([100, 70], [6, 1], kv=2, width=64, page=32)
    page, width = run.page, run.width
    q = run.random(4, 5)
    want = attend(run, q)
    scales = run.cache.data[:, :, page * width:].contiguous().view(torch.float32).reshape(-1, 2, 2, page)
    for b, n in enumerate(run.len):
        at = n - 1                                                      # the newest token, seen by the last row only
        for j, value in ((at, NAN), (at + 1, INF), (at + 2, NAN)):
            p = run.table[b, j // page]
            if p >= 0:
                scales[p, :, :, j % page] = value
    owned = set(run.table.flatten().tolist())
    for p in range(run.cache.pages):
        if p not in owned:
            scales[p] = NAN
    run.cache.data[:, :, page * width:] = scales.reshape(-1, 2, 2 * page).view(torch.uint8)
    y = attend(run, q)
    assert bool(y[5].isnan().all()) and bool(y[6].isnan().all())
    assert torch.equal(y[:5], want[:5])


def test_attend_queries_with_an_infinity_or_a_nan():
    """They make their own head of their own row NaN."""
    run = Run([100, 70], [6, 1], kv=2, width=128)
    q = run.random(4, 5)
    want = attend(run, q)
    q[1, 2, 5], q[4, 0, 0], q[6, 3, 127] = INF, NAN, -INF
    y = attend(run, q)
    bad = torch.zeros(7, 4, dtype=torch.bool, device="cuda")
    bad[1, 2] = bad[4, 0] = bad[6, 3] = True
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], want[~bad])


def test_attend_strides():
    run = Run([90, 33], [40, 2], kv=2, width=128)
    q = run.random(8, 5)
    want = attend(run, q)
    wide = torch.zeros(run.rows, 3, 8, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 0] = q
    H.attend_tokens(wide[:, 0], run.cache, run.table, run.lengths, run.starts, out=wide[:, 1])
    outside = q.transpose(0, 1).contiguous().transpose(0, 1)
    y = torch.empty_like(outside)
    H.attend_tokens(outside, run.cache, run.table, run.lengths, run.starts, out=y)
    odd = torch.zeros(run.rows, 8, 131, dtype=torch.bfloat16, device="cuda")
    odd[:, :, 1:129] = q
    z = attend(run, odd[:, :, 1:129])
    table = torch.full((2, 50), -1, dtype=torch.int32, device="cuda")[:, 7:7 + run.table.shape[1]]
    table.copy_(run.table)
    w = H.attend_tokens(q, run.cache, table, run.lengths, run.starts)
    finish()
    assert torch.equal(wide[:, 1], want) and torch.equal(y, want) and torch.equal(z, want) and torch.equal(w, want)
    assert bool((wide[:, 2] == 0).all()) and torch.equal(wide[:, 0], q)
    first = q[:1].expand(run.rows, -1, -1)
    assert torch.equal(attend(run, first), attend(run, first.contiguous()))


# Many queries per sequence and bf16: another kernel. It rounds code times scale to fp16 as well, of keys (as q is) and of
# values (as w v is): variances twice as large, deviations sqrt(2) times.
MANY = 2 ** 0.5


def some(run, n, seed=0):
    """Rows to compare: the first and last of every sequence, and n others."""
    ends, at = set(), 0
    for m in run.new:
        if m:
            ends |= {at, at + m - 1}
        at += m
    return ends | set(np.random.default_rng(seed).integers(0, at, n).tolist())


@pytest.mark.parametrize("width,hb,page", [(64, 64, 16), (64, 1, 64), (64, 8, 32), (128, 128, 64), (128, 64, 16), (128, 2, 32), (128, 1, 64)])
@pytest.mark.parametrize("kv,group", [(16, 2), (12, 7), (40, 1)])
def test_attend_many_columns(width, hb, page, kv, group):
    """Columns below, at and above a tile's, last tiles cut, sequences without tokens, without keys, with more rows than tokens."""
    lengths = [64, 40, 130, 0, 5, 260, 127, 65, 700]
    run = Run(lengths, [64, 3, 130, 0, 9, 1, 127, 64, 37], kv=kv, width=width, page=page, hb=hb)
    q = run.random(kv * group, 5)
    check_attend(run, q, attend(run, q), rows=some(run, 60), more=MANY)


@pytest.mark.parametrize("width", [64, 128])
def test_attend_long_prompts(width):
    run = Run([1900, 1111], [1500, 1111], kv=8, width=width)
    q = run.random(32, 5)
    check_attend(run, q, attend(run, q), rows=some(run, 30), more=MANY)


@pytest.mark.parametrize("scale", [0.0, 1e-3, 0.7, -0.3, 8.0])
def test_attend_many_columns_scales(scale):
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=64)
    q = run.random(64, 5)
    check_attend(run, q, attend(run, q, scale=scale), scale, rows=some(run, 40), more=MANY)


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e4, 1e30])
def test_attend_many_columns_scales_of_any_size(size):
    """Of values times size; of both growing from token to token, so that later ones raise what the first were brought to."""
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=128)
    at = run.page * run.width
    scales = run.cache.data[:, :, at:].contiguous().view(torch.float32).reshape(-1, 16, 2, run.page)
    scales[:, :, 1] *= size
    for b, n in enumerate(run.len):
        for j in range(n):
            scales[run.table[b, j // run.page], :, 1, j % run.page] *= 1.05 ** (j - n)
    run.cache.data[:, :, at:] = scales.reshape(-1, 16, 2 * run.page).view(torch.uint8)
    q = run.random(64, 5)
    y = attend(run, q)
    rows = some(run, 40)
    ref, sd = reference(run, q, rows=rows)
    tol = 8 * MANY * sd + 2.0 ** -8 * 1.01 * ref.abs() + 2.0 ** -130
    assert float(((y.double().cpu() - ref).abs() / tol)[sorted(rows)].max()) <= 1


def test_attend_many_columns_pages_that_are_none():
    run = Run([200, 333, 90, 40], [60, 40, 90, 48], kv=16, width=64, page=16)
    run.table[0, 3], run.table[1, 0], run.table[1, 20] = -1, 1 << 30, run.cache.pages
    run.table[2, :] = -1
    q = run.random(64, 5)
    y = attend(run, q)
    check_attend(run, q, y, rows=some(run, 60), more=MANY)
    assert bool((y[100:190] == 0).all()) and bool((y[190:198] == 0).all()) and bool((y[198:] != 0).any())


def test_attend_many_columns_what_a_row_does_not_see():
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=64, page=32)
    page, width = run.page, run.width
    q = run.random(64, 5)
    want = attend(run, q)
    scales = run.cache.data[:, :, page * width:].contiguous().view(torch.float32).reshape(-1, 16, 2, page)
    first = {0: 150, 1: 332, 2: 1, 3: 64}                               # the first token that is NaN, by sequence (3: none)
    for b, n in enumerate(run.len):
        for part, j in ((0, first[b]), (1, first[b] + 1), (1, n), (0, n + 1)):
            if j >= first[b] and j // page < run.table.shape[1] and run.table[b, j // page] >= 0:
                scales[run.table[b, j // page], :, part, j % page] = NAN
    run.cache.data[:, :, page * width:] = scales.reshape(-1, 16, 2 * page).view(torch.uint8)
    y = attend(run, q)
    for r, b, p in run.places():
        if p >= first[b]:
            assert bool(y[r].isnan().all())
        else:
            assert torch.equal(y[r], want[r])


def test_attend_many_columns_queries_with_an_infinity_or_a_nan():
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=128)
    q = run.random(64, 5)
    want = attend(run, q)
    bad = torch.zeros(254, 64, dtype=torch.bool, device="cuda")
    for r, h, d, v in ((1, 2, 5, INF), (100, 0, 0, NAN), (253, 63, 127, -INF)):
        q[r, h, d], bad[r, h] = v, True
    y = attend(run, q)
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], want[~bad])


def test_attend_many_columns_strides_and_rows_of_no_sequence():
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=64)
    q = run.random(32, 5)
    want = attend(run, q)
    odd, out = torch.zeros(260, 32, 67, dtype=torch.bfloat16, device="cuda"), torch.full((260, 32, 67), 7.0, dtype=torch.bfloat16, device="cuda")
    odd[3:257, :, 1:65] = q
    H.attend_tokens(odd[:, :, 1:65], run.cache, run.table, run.lengths, run.starts + 3, out=out[:, :, 2:66])
    outside = q.transpose(0, 1).contiguous().transpose(0, 1)
    y = torch.empty_like(outside)
    H.attend_tokens(outside, run.cache, run.table, run.lengths, run.starts, out=y)
    finish()
    assert torch.equal(out[3:257, :, 2:66], want) and torch.equal(y, want)
    out[3:257, :, 2:66] = 7
    assert bool((out == 7).all())


def test_attend_many_columns_twice_and_in_a_graph():
    run = Run([200, 333, 90, 64], [60, 40, 90, 64], kv=16, width=128)
    q, p = run.random(64, 5), run.random(64, 6)
    want = attend(run, q), attend(run, p)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [(H.attend_tokens(q, run.cache, run.table, run.lengths, run.starts, stream=a),
            H.attend_tokens(p, run.cache, run.table, run.lengths, run.starts, stream=b)) for _ in range(10)]
    finish()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = H.attend_tokens(q, run.cache, run.table, run.lengths, run.starts)
    for src, ref in ((p, want[1]), (q.clone(), want[0])):
        q.copy_(src)
        graph.replay()
        finish()
        assert torch.equal(y, ref)


def test_attend_twice_and_on_two_streams():
    run = Run([3000, 700, 64, 1], [1, 1, 1, 1], kv=4, width=128, one_each=True)
    q, p = run.random(16, 5), run.random(16, 6)
    want_q, want_p = attend(run, q), attend(run, p)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    a.wait_stream(torch.cuda.current_stream())
    b.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        got.append((H.attend_tokens(q, run.cache, run.table, run.lengths, stream=a),
                    H.attend_tokens(p, run.cache, run.table, run.lengths, stream=b)))
    finish()
    assert all(torch.equal(x, want_q) and torch.equal(y, want_p) for x, y in got)


def test_attend_pages_beyond_4_gb():
    run = Run([200], [1], kv=1, width=128, one_each=True)
    q = run.random(4, 5)
    want = attend(run, q)
    pages = 600_000
    cache = H.TokenCache.empty(pages, 1, 128, page=64, hb=128)
    table = torch.tensor([[pages - 1, 5, pages - 7, 590_000]], dtype=torch.int32, device="cuda")
    for i in range(4):
        cache.data[table[0, i]] = run.cache.data[run.table[0, i]]
    y = H.attend_tokens(q, cache, table, run.lengths)
    finish()
    assert torch.equal(y, want)


def test_a_step_in_a_graph():
    """Append and attend captured once and replayed as the sequences grow: the same as calls of their own."""
    lengths, steps = [60, 1, 126], 6
    run, eager = (Run([n + steps for n in lengths], [1] * 3, kv=2, width=64, page=16, one_each=True) for _ in range(2))
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    k, v, q = run.random(2, 5), run.random(2, 6), run.random(8, 7)

    def step(r):
        H.append_tokens(r.cache, k, v, r.table, at)
        return H.attend_tokens(q, r.cache, r.table, at)

    before = run.cache.data.clone()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(run)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = step(run)
    torch.cuda.synchronize()
    run.cache.data.copy_(before)
    for i in range(steps):
        for x, seed in ((k, 10), (v, 20), (q, 30)):
            x.copy_(torch.randn(x.shape, generator=gen(seed + i), device="cuda"))
        at += 1
        graph.replay()
        want = step(eager)
        finish()
        assert torch.equal(y, want) and torch.equal(run.cache.data, eager.cache.data)
    eager.len = [n + steps for n in lengths]
    check_attend(eager, q, want)


def test_refusals():
    run = Run([40, 9], [3, 2], kv=2, width=64)
    q, k = run.random(4, 5), run.random(2, 6)
    ok = (run.cache, run.table, run.lengths, run.starts)
    for bad in (lambda: H.attend_tokens(q.float(), *ok), lambda: H.attend_tokens(q[:, :3], *ok),
                lambda: H.attend_tokens(q[:, :, :32], *ok), lambda: H.attend_tokens(q, *ok[:3]),
                lambda: H.attend_tokens(q, *ok, out=q), lambda: H.attend_tokens(q, *ok, out=torch.empty_like(q).half()),
                lambda: H.attend_tokens(q, run.cache, run.table.long(), run.lengths, run.starts),
                lambda: H.attend_tokens(q, run.cache, run.table, run.lengths[:1], run.starts),
                lambda: H.attend_tokens(q, run.cache, run.table, run.lengths, run.starts[:2]),
                lambda: H.attend_tokens(q.cpu(), *ok), lambda: H.attend_tokens(q, *ok, scale=INF),
                lambda: H.attend_tokens(q, *ok, out=torch.empty_like(q[:1]).expand(5, -1, -1)),
                lambda: H.append_tokens(run.cache, k, k.half(), *ok[1:]), lambda: H.append_tokens(run.cache, k, k[1:], *ok[1:]),
                lambda: H.append_tokens(run.cache, k.double(), k.double(), *ok[1:]),
                lambda: H.append_tokens(run.cache, k[:, :1], k[:, :1], *ok[1:]),
                lambda: H.TokenCache(run.cache.data.float()), lambda: H.TokenCache(run.cache.data[:, :, 1:]),
                lambda: H.TokenCache(run.cache.data, page=48), lambda: H.TokenCache(run.cache.data, hb=128),
                lambda: H.TokenCache.empty(2, 2, 96)):
        with pytest.raises((ValueError, H.HatqError)):
            bad()
    finish()


def test_attend_many_sequences():
    """More sequences than a warp has lanes, several a lane, of all lengths down to none."""
    lengths = [(37 * i) % 190 for i in range(700)]
    run = Run(lengths, [1] * 700, kv=2, width=64, page=16, one_each=True)
    q = run.random(10, 5)
    check_attend(run, q, attend(run, q), rows=some(run, 100))
    new = [min(n, i % 3) for i, n in enumerate(lengths)]
    run = Run(lengths, new, kv=2, width=64, page=16)
    q = run.random(4, 5)
    check_attend(run, q, attend(run, q), rows=some(run, 100))


def test_attend_parts_of_many_sequences():
    """The same in equal parts: more segments than a CTA each would be worth, some sequences much longer."""
    lengths = [700 if i % 50 == 3 else (7 * i) % 30 for i in range(500)]
    run = Run(lengths, [1] * 500, kv=8, width=128, page=64, one_each=True)
    q = run.random(16, 5)
    check_attend(run, q, attend(run, q), rows=some(run, 60) | {3, 53, 103})


def test_append_many_sequences():
    """More offsets than are looked at at a time, some sequences without rows, one head: eight rows of a warp."""
    new = [(i * i) % 4 for i in range(900)]
    run = Run([m + i % 60 for i, m in enumerate(new)], new, kv=1, width=64, page=16)
    check_append(run, run.random(1, 5), run.random(1, 6))


# ------------------------------------------------------------------ scales far from one another

# A few queries per sequence; many, which bf16 queries take to the other kernel.
FEW = dict(lengths=[200, 333], new=[3, 1], kv=2, width=64)
MANY_COLUMNS = dict(lengths=[200, 333, 90, 64], new=[60, 40, 90, 64], kv=16, width=64)
SHAPES = [(FEW, 4, "bf16"), (FEW, 4, "f16"), (dict(FEW, width=128), 6, "bf16"), (MANY_COLUMNS, 64, "f16"), (MANY_COLUMNS, 64, "bf16"),
          (dict(MANY_COLUMNS, width=128, page=16), 64, "bf16")]


def scales_of(run):
    """Scales of the cache [pages][kv][2][page]: keys', values'."""
    return run.cache.data[:, :, run.page * run.width:].contiguous().view(torch.float32).reshape(-1, run.kv, 2, run.page)


def put_scales(run, scales):
    run.cache.data[:, :, run.page * run.width:] = scales.reshape(-1, run.kv, 2 * run.page).view(torch.uint8)


def put_codes(run, part, b, j, code):
    """One code for all of a token's keys (part 0) or values."""
    at = (part * run.page + j % run.page) * run.width // 2
    run.cache.data[run.table[b, j // run.page], :, at:at + run.width // 2] = 17 * (code + 8)


def some_rows(run):
    return list(range(run.rows)) if run.rows < 20 else sorted(some(run, 25))


def check_within(run, q, y, ref, sd, rows):
    """As check_attend does, with nothing added to the bound but what the type itself cannot hold (bf16: outputs of any
    size count). The other kernel's deviations for all."""
    tol = 8 * MANY * sd + torch.finfo(q.dtype).eps / 2 * 1.01 * ref.abs() + (2.0 ** -24 if q.dtype == torch.float16 else 2.0 ** -130)
    assert len(rows) and float(((y.double().cpu() - ref).abs() / tol)[rows].nan_to_num(nan=INF).max()) <= 1


@pytest.mark.parametrize("part", ["keys", "values"])
@pytest.mark.parametrize("size", [2.0 ** 9, 2.0 ** 13, 2.0 ** 20, 2.0 ** 33, 2.0 ** 90, INF])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_a_large_scale_that_a_row_does_not_see(shape, heads, dtype, size, part):
    """The newest token of every sequence, which only the last row sees."""
    run = Run(**shape, dtype=dtype)
    q = run.random(heads, 5)
    last = set((np.cumsum(run.new) - 1).tolist())
    rows = [r for r in some_rows(run) if r not in last]
    ref, sd = reference(run, q, rows=rows)
    scales = scales_of(run)
    for b, n in enumerate(run.len):
        scales[run.table[b, (n - 1) // run.page], :, 0 if part == "keys" else 1, (n - 1) % run.page] *= size
    put_scales(run, scales)
    check_within(run, q, attend(run, q), ref, sd, rows)


@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_values_of_nothing_say_nothing(shape, heads, dtype, size):
    """Tokens whose value codes are all 0, single ones and the whole first chunk, whatever their scale: as with a scale of 0."""
    run = Run(**shape, dtype=dtype)
    q = run.random(heads, 5)
    rows = some_rows(run)
    scales = scales_of(run)
    for b, n in enumerate(run.len):
        for j in {0, 40, n - 1} | set(range(64) if b == 1 else ()):
            put_codes(run, 1, b, j, 0)
            scales[run.table[b, j // run.page], :, 1, j % run.page] = 0
    put_scales(run, scales)
    ref, sd = reference(run, q, rows=rows)
    put_scales(run, torch.where(scales == 0, size, scales))
    check_within(run, q, attend(run, q), ref, sd, rows)


@pytest.mark.parametrize("size", [4.0, 10.0, 20.0, 40.0, 100.0])
@pytest.mark.parametrize("width,hb,page,group", [(64, 1, 16, 4), (128, 128, 64, 1), (256, 1, 16, 4), (256, 256, 16, 1)])
@pytest.mark.parametrize("seed", [3, 26, 34, 56])
def test_attend_values_of_nothing_among_the_others(width, hb, page, group, seed, size):
    """Two in five tokens have value codes of 0 and scales some times those of the others: too near them to raise a maximum."""
    lengths = [559, 60, 132, 490, 32, 400, 375, 68]
    run = Run(lengths, [1] * 8, kv=2, width=width, page=page, hb=hb, seed=seed, one_each=True)
    pick = np.random.default_rng(seed)
    scales = scales_of(run)
    for b, n in enumerate(lengths):
        for j in range(1, n):
            if pick.random() < 0.4:
                put_codes(run, 1, b, j, 0)
                scales[run.table[b, j // page], :, 1, j % page] = 0
    put_scales(run, scales)
    q = run.random(2 * group, 5)
    ref, sd = reference(run, q, 0.05)                                   # (small logits: the others keep weights of their own)
    put_scales(run, torch.where(scales == 0, size, scales))
    check_within(run, q, attend(run, q, scale=0.05), ref, sd, list(range(8)))


@pytest.mark.parametrize("size", [0.0, 2.0 ** -100, 1.0, 2.0 ** 100])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_values_of_nothing_alone(shape, heads, dtype, size):
    """All value codes are 0, or (size 0) all value scales: zeros."""
    run = Run(**shape, dtype=dtype)
    half = run.page * run.width // 2
    if size:
        run.cache.data[:, :, half:2 * half] = 0x88
    scales = scales_of(run)
    scales[:, :, 1] *= size
    put_scales(run, scales)
    assert bool((attend(run, run.random(heads, 5)) == 0).all())


@pytest.mark.parametrize("shape,heads", [(FEW, 4), (MANY_COLUMNS, 64)])
def test_attend_zeros_appended_among_small_values(shape, heads):
    """Append gives a row of zeros a scale of 1 / sqrt(hb): the values of 1e-12 beside it stay what they are."""
    run = Run(**shape)
    new = dict(shape, new=shape["lengths"])                             # all tokens go in at once
    fill = Run(**new)
    k, v = fill.random(run.kv, 5), fill.random(run.kv, 6) * 1e-12
    at = 0
    for n in run.len:
        v[at + 7], v[at + n - 1] = 0, 0
        at += n
    H.append_tokens(run.cache, k, v, run.table, run.lengths, fill.starts)
    q = run.random(heads, 8)
    rows = some_rows(run)
    y = attend(run, q)
    scales = scales_of(run)
    scales[:, :, 1] = torch.where(scales[:, :, 1] == 1 / math.sqrt(run.hb), 0.0, scales[:, :, 1])
    put_scales(run, scales)
    ref, sd = reference(run, q, rows=rows)
    check_within(run, q, y, ref, sd, rows)


@pytest.mark.parametrize("part", ["keys", "values"])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_scales_of_many_sizes_that_rows_see(shape, heads, dtype, part):
    """Value scales spread over 2^60 (fp16: up to 2^10, what its outputs hold), key scales over 2^40 down from 1."""
    run = Run(**shape, dtype=dtype)
    q = run.random(heads, 5)
    scales = scales_of(run)
    u = torch.rand(scales.shape[:2] + scales.shape[3:], generator=gen(9), device="cuda")
    if part == "keys":
        scales[:, :, 0] *= 2.0 ** (-40 * u)
    else:
        scales[:, :, 1] *= 2.0 ** (60 * u - (30 if dtype == "bf16" else 50))
    put_scales(run, scales)
    rows = some_rows(run)
    ref, sd = reference(run, q, rows=rows)
    check_within(run, q, attend(run, q), ref, sd, rows)


@pytest.mark.parametrize("size", [2.0 ** -105, 2.0 ** 107])
@pytest.mark.parametrize("shape,heads,dtype", [x for x in SHAPES if x[2] == "bf16"])
def test_attend_value_scales_at_the_ends_of_their_range(shape, heads, dtype, size):
    run = Run(**shape, dtype=dtype)
    q = run.random(heads, 5)
    scales = scales_of(run)
    scales[:, :, 1] *= size
    put_scales(run, scales)
    rows = some_rows(run)
    ref, sd = reference(run, q, rows=rows)
    check_within(run, q, attend(run, q), ref, sd, rows)


@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_large_values_of_no_weight(shape, heads, dtype, first):
    """Half of the tokens weigh 2^-80 of the others, each, and have values of 2^40 (fp16: 2^12) times theirs: nothing of
    them is in the output, and what there is of the others is whole. Equal keys, so that a common error of their logits
    cancels; the light half comes first or last, or in turns of 5."""
    for turns in (False, True):
        run = Run(**shape, hb=1, dtype=dtype)
        q = torch.ones_like(run.random(heads, 5))
        scales = scales_of(run)
        scales[:, :, 0] = 4 / run.width ** 0.5                           # logits of +-28
        for b, n in enumerate(run.len):
            for j in range(n):
                light = (j // 5 % 2 == 0) if turns else (j < n // 2) == first
                put_codes(run, 0, b, j, -7 if light else 7)
                if light:
                    scales[run.table[b, j // run.page], :, 1, j % run.page] *= 2.0 ** (40 if dtype == "bf16" else 12)
        put_scales(run, scales)
        rows = some_rows(run)
        ref, sd = reference(run, q, rows=rows)
        check_within(run, q, attend(run, q), ref, sd, rows)


@pytest.mark.parametrize("scale", [1e31, -1e31])
@pytest.mark.parametrize("shape,heads,dtype,size", [(*x, size) for x in SHAPES for size in ((1.0, 2.0 ** -60, 2.0 ** 60) if x[2] == "bf16" else (1.0,))])
def test_attend_logits_far_from_zero(shape, heads, dtype, scale, size):
    """A row that sees one token has its value, however low or high the logit: no magnitude stands for "no token". (fp16:
    values that it holds.)"""
    run = Run(**dict(shape, lengths=[max(m, 1) for m in shape["new"]]), dtype=dtype)
    scales = scales_of(run)
    scales[:, :, 1] *= size
    put_scales(run, scales)
    q = run.random(heads, 5)
    rows = [r for r, _, p in run.places() if p == 0]
    ref, sd = reference(run, q, rows=rows)                              # (one weight of 1: of any scale)
    check_within(run, q, attend(run, q, scale=scale), ref, sd, rows)


@pytest.mark.parametrize("spread", [0, 20])
@pytest.mark.parametrize("logit", [3e3, -2e4, 3e6, -1e9, 1e20, -1e30])
@pytest.mark.parametrize("shape,heads,dtype", SHAPES)
def test_attend_equal_logits_of_any_size(shape, heads, dtype, logit, spread):
    """Equal keys: the average of the values that a row sees, as with a scale of 0. (fp16: spread by 2^10, as its outputs are.)"""
    run = Run(**shape, hb=1, dtype=dtype)
    q = torch.ones_like(run.random(heads, 5))
    for b, n in enumerate(run.len):
        for j in range(n):
            put_codes(run, 0, b, j, 7)
    scales = scales_of(run)
    scales[:, :, 0] = 1 / 7
    if spread:
        u = torch.rand(scales.shape[:2] + scales.shape[3:], generator=gen(9), device="cuda")
        scales[:, :, 1] *= 2.0 ** ((2 * u - 1) * (spread if dtype == "bf16" else 5))
    put_scales(run, scales)
    rows = some_rows(run)
    ref, sd = reference(run, q, 0.0, rows=rows)
    check_within(run, q, attend(run, q, scale=logit / run.width), ref, sd, rows)
