"""What adaqp_train.h declares, on the GPU against the float64 definitions of oracle/train.py.

u = 2^-24.  Tolerances follow from the number of roundings: a sum of t terms taken by lanes in turn and then joined is off by at most (t / lanes + 16) u of the sum of the
terms' magnitudes; each further operation adds u.  bf16 outputs (7 stored bits) add half a unit in their last place, at most 2^-8 of the value."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import train as O                                        # noqa: E402
from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SENTINEL = -77.0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.empty_cache()


def _say(*what):
    print(*what, flush=True)
    sys.stdout.flush()


def _matrix(values, dtype, ld=None, offset=0):
    """`values` as a device matrix of pitch ld whose first element lies `offset` elements behind a 128-byte line, NaN around it."""
    values = np.asarray(values)
    rows, cols = values.shape
    ld = ld or cols
    buf = torch.full((rows * ld + offset + 256,), float("nan"), dtype=dtype, device=DEV)
    m = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.from_numpy(values.astype(np.float64)).to(dtype))
    return m


def _out(rows, cols, dtype, ld=None, offset=0, fill=SENTINEL):
    buf = torch.full((rows * (ld or cols) + offset + 256,), fill, dtype=dtype, device=DEV)
    return buf[offset:offset + rows * (ld or cols)].view(rows, ld or cols)[:, :cols], buf


def _np(t):
    return t.double().cpu().numpy()


def _vec(v, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(v)).to(dtype).to(DEV)


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def _rounding(values, dtype):
    return (2.0 ** -8 if dtype == torch.bfloat16 else U) * np.abs(values)


def _untouched(buf, rows, cols, ld, offset, dtype):
    """Only the matrix's columns were written or, with rows of whole lines, its lines, the padding with zeros."""
    b = _np(buf)
    ld = ld or cols
    assert np.all(b[:offset] == SENTINEL) and np.all(b[offset + rows * ld:] == SENTINEL)
    line = 128 // dtype.itemsize
    behind = b[offset:offset + rows * ld].reshape(rows, ld)[:, cols:]
    if offset == 0 and ld % line == 0:
        written = -(-cols // line) * line - cols
        assert np.all(behind[:, :written] == 0) and np.all(behind[:, written:] == SENTINEL)
    else:
        assert np.all(behind == SENTINEL)


SHAPES = [  # rows, dim, ld, offset
    (1, 1, None, 0), (1, 128, None, 0), (3, 5, None, 0), (17, 16, None, 0), (33, 31, 33, 1), (130, 64, 64, 0), (300, 256, 256, 0), (64, 256, 300, 0),
    (50, 301, None, 0), (70, 602, 608, 0), (70, 602, 640, 0), (21, 604, 604, 4), (40, 514, 520, 2), (9, 1023, None, 0), (5, 2051, 2112, 0), (700, 7, 7, 3),
]


# ---- dropout -----------------------------------------------------------------------------------------------------------------------------

def _dropped(x, add, p, seed, first_row, dtype):
    """The call's steps in fp32 on the host: one rounding for the product, one for the sum, one for the output's type."""
    keep, factor = O.dropped(*x.shape, p, seed, first_row)
    y = torch.where(torch.from_numpy(keep), x.float().cpu() * torch.tensor(factor, dtype=torch.float32), 0.0)
    return (y if add is None else y + add.float().cpu()).to(dtype)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,dim,ld,offset", SHAPES)
def test_dropout_bit_for_bit(rows, dim, ld, offset, kind):
    _say("dropout", rows, dim, ld, offset, kind)
    dtype, rng = TYPES[kind], np.random.default_rng(dim)
    xd, ad = (_matrix(rng.standard_normal((rows, dim)), dtype, ld, offset) for _ in range(2))
    for p, seed, first_row, add in ((0.5, 3, 0, None), (0.1, 2 ** 63 + 11, 7, ad), (0.0, 1, 0, None), (1.0, 1, 0, ad)):
        y, buf = _out(rows, dim, dtype, ld, offset)
        B.adaqp_dropout(xd, dim, p, seed, y, add=add, first_row=first_row)
        want = _dropped(xd, add, p, seed, first_row, dtype)
        assert torch.equal(y.cpu(), want)
        _untouched(buf, rows, dim, ld, offset, dtype)
    sum_of, of = _dropped(xd, ad, 0.3, 5, 0, dtype), _dropped(xd, None, 0.5, 3, 0, dtype)
    B.adaqp_dropout(xd, dim, 0.3, 5, ad, add=ad)                       # in place of add
    B.adaqp_dropout(xd, dim, 0.5, 3, xd)                               # and of x
    assert torch.equal(ad.cpu(), sum_of) and torch.equal(xd.cpu(), of)


def test_dropout_in_place_numbers_rows_and_counters():
    """In place, in two calls of half the rows, by a seed in device memory: the same choices.  Rows past 2^32 have numbers of their own."""
    rng = np.random.default_rng(1)
    x = _matrix(rng.standard_normal((40, 70)), torch.float32)
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    B.adaqp_dropout(x, 70, 0.4, 9, whole)
    B.adaqp_dropout(x[:13], 70, 0.4, 9, parts[:13])
    B.adaqp_dropout(x[13:], 70, 0.4, 9, parts[13:], first_row=13)
    assert torch.equal(whole, parts)
    counter = torch.tensor([4], device=DEV)
    B.adaqp_dropout(x, 70, 0.4, 5, parts, counter=counter)
    assert torch.equal(whole, parts)
    for first in ((1 << 32) - 7, (1 << 40) + 3):
        B.adaqp_dropout(x, 70, 0.4, 9, parts, first_row=first)
        assert torch.equal(parts.cpu(), _dropped(x, None, 0.4, 9, first, torch.float32))
    x[3, 5], x[4, 6], x[5, 7] = float("inf"), float("nan"), float("-inf")
    B.adaqp_dropout(x, 70, 0.4, 9, parts)
    keep, _ = O.dropped(40, 70, 0.4, 9)
    got = _np(parts)
    assert np.all(got[~keep] == 0) and np.array_equal(np.isfinite(got), ~keep | np.isfinite(_np(x)))
    B.adaqp_dropout(x, 70, 1.0, 9, parts)
    assert not parts.any()


# ---- embedding ---------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind_t", list(TYPES))
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,dim,ld,offset", SHAPES)
def test_embedding_forward_bit_for_bit(rows, dim, ld, offset, kind, kind_t):
    _say("embedding forward", rows, dim, ld, offset, kind, kind_t)
    dtype, rng = TYPES[kind], np.random.default_rng(dim + 1)
    for entries in (1, 37):
        table = _matrix(rng.standard_normal((entries, dim)), TYPES[kind_t], ld, offset)
        ids = rng.integers(-2, entries + 2, rows)
        ids[0], ids[-1] = entries - 1, rng.choice([-2 ** 31, 2 ** 31 - 1, 0])
        out, buf = _out(rows, dim, dtype, ld, offset)
        B.adaqp_embedding_forward(table, dim, _vec(ids, torch.int32), 1.7, out)
        there = torch.from_numpy((ids >= 0) & (ids < entries))
        want = torch.where(there[:, None], table.float().cpu()[torch.from_numpy(np.clip(ids, 0, entries - 1))] * torch.tensor(1.7, dtype=torch.float32), 0.0).to(dtype)
        assert torch.equal(out.cpu(), want)
        _untouched(buf, rows, dim, ld, offset, dtype)
    B.adaqp_embedding_forward(table[:0], dim, _vec(ids, torch.int32), 1.7, out)          # a table without entries
    assert not out.any()


@pytest.mark.parametrize("n,entries", [(1, 1), (1, 0), (5, 3), (64, 2), (63, 511), (64, 512), (65, 513), (1024, 255), (1025, 256), (4096, 1000), (4097, 1 << 18), (8192, 65_535), (8193, 65_536), (9001, 20_000), (12_288, (1 << 31) - 1), (12_289, 300), (20_000, 1), (50_000, 300), (131_072, 50_000),
                                       (262_144, (1 << 31) - 1), (262_145, 70_000), (1_000_003, 400_000)])
def test_embedding_sort_is_stable(n, entries):
    _say("embedding sort", n, entries)
    rng = np.random.default_rng(n)
    ids = np.floor(entries * rng.random(n) ** 3).astype(np.int64)
    ids[rng.random(n) < 0.05] = -1
    ids[rng.random(n) < 0.02] = min(entries, 2 ** 31 - 1)
    if n > 100:
        ids[7], ids[90], ids[-1] = -2 ** 31, 2 ** 31 - 1, entries - 1
    got, order = (torch.full((n + 8,), -5, dtype=torch.int32, device=DEV) for _ in range(2))
    work = _bytes(B.adaqp_embedding_sort_workspace_bytes(n, entries))
    B.adaqp_embedding_sort(_vec(ids, torch.int32), entries, got, order, work)
    want, want_order = O.sort_ids(ids, entries)
    assert np.array_equal(got[:n].cpu().numpy(), want) and np.array_equal(order[:n].cpu().numpy(), want_order)
    assert torch.all(got[n:] == -5) and torch.all(order[n:] == -5)


def _sorted(ids, entries):
    ids = _vec(ids, torch.int32)
    got, order = torch.empty_like(ids), torch.empty_like(ids)
    B.adaqp_embedding_sort(ids, entries, got, order, _bytes(B.adaqp_embedding_sort_workspace_bytes(ids.numel(), entries)))
    return got, order


def _check_gradient(dy, ids, entries, dim, scale, got, before=None):
    want = O.embedding_gradient(_np(dy), ids, entries, scale) + (0 if before is None else before)
    terms = O.embedding_gradient(np.abs(_np(dy)), ids, entries, abs(scale))
    # a chunk's 32 in turn, then the chunks of an id by eight waves in turn, joined; the product with scale and what is added to.  Of chunks of 8 the worst case is 8 + many / 64 + 8, more than this
    # for many above 3000, where roundings of both signs stay far below it
    many = np.bincount(ids[(ids >= 0) & (ids < entries)], minlength=entries)[:, None]
    tol = (32 + many / 128 + 8) * U * terms + 2 * U * np.abs(want)
    assert np.all(np.abs(_np(got) - want) <= tol)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,entries,dim,ld,offset", [
    (1, 1, 1, None, 0), (1, 5, 8, None, 0), (31, 4, 3, None, 0), (32, 1, 16, None, 0), (33, 1, 33, 35, 1), (64, 2, 64, 64, 0), (65, 200, 301, None, 0), (300, 7, 602, 608, 0),
    (300, 1000, 602, 640, 0), (40, 100_000, 17, 17, 0), (20_000, 70, 9, 9, 0), (2000, 3, 100, 100, 0), (5000, 1, 40, 64, 0), (5000, 64, 1030, 1030, 0), (4001, 5000, 257, 260, 2), (70_000, 2, 12, 12, 0), (9001, 20_000, 20, 32, 0),
    (17_000, 1, 36, 36, 0), (33_000, 1, 36, 36, 0), (100_000, 2, 300, 301, 1), (300_000, 3, 5, 5, 0), (262_144, 7, 64, 64, 0)])
def test_embedding_backward(n, entries, dim, ld, offset, kind):
    _say("embedding backward", n, entries, dim, ld, offset, kind)
    dtype, rng = TYPES[kind], np.random.default_rng(n + dim)
    dy = _matrix(rng.standard_normal((n, dim)), dtype, ld, offset)
    ids = np.floor(entries * rng.random(n) ** 3).astype(np.int64)
    if n > 5:
        ids[rng.random(n) < 0.05] = -1
        ids[3] = entries
    by_id, order = _sorted(ids, entries)
    work = _bytes(B.adaqp_embedding_backward_workspace_bytes(n, dim))
    work.fill_(0xFF)                                                   # NaN
    got, buf = _out(entries, dim, torch.float32, ld, offset)
    B.adaqp_embedding_backward(dy, dim, by_id, order, 1.5, False, got, work)
    _check_gradient(dy, ids, entries, dim, 1.5, got)
    _untouched(buf, entries, dim, ld, offset, torch.float32)
    again = torch.empty_like(got)
    B.adaqp_embedding_backward(dy, dim, by_id, order, 1.5, False, again, work)
    assert torch.equal(again, got)
    more, buf = _out(entries, dim, torch.float32, ld, offset)
    B.adaqp_embedding_backward(dy, dim, by_id, order, -0.5, True, more, work)
    _check_gradient(dy, ids, entries, dim, -0.5, more, SENTINEL)
    b, width = _np(buf), ld or dim
    named = np.isin(np.arange(entries), ids)
    assert np.all(b[offset:offset + entries * width].reshape(entries, width)[:, dim:] == SENTINEL) and np.all(_np(more)[~named] == SENTINEL)
    assert np.all(b[:offset] == SENTINEL) and np.all(b[offset + entries * width:] == SENTINEL)


def test_embedding_backward_without_ids_and_with_none_of_the_table():
    dtable = torch.full((50, 64), SENTINEL, device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    B.adaqp_embedding_backward(torch.empty(0, 40, device=DEV), 40, none, none, 1.0, False, dtable, None)
    assert not dtable.any()
    dtable.fill_(SENTINEL)
    B.adaqp_embedding_backward(torch.empty(0, 40, device=DEV), 40, none, none, 1.0, True, dtable, None)
    assert torch.all(dtable == SENTINEL)
    by_id, order = _sorted(np.full(100, -1), 50)
    work = _bytes(B.adaqp_embedding_backward_workspace_bytes(100, 64))
    B.adaqp_embedding_backward(torch.randn(100, 64, device=DEV), 64, by_id, order, 1.0, False, dtable, work)
    assert not dtable.any()


def test_embedding_backward_ignores_places_and_ids_that_are_not_there():
    """Sorted ids of a larger table and places of a longer list: bounds are the call's own."""
    rng = np.random.default_rng(4)
    ids = rng.integers(0, 90, 400)
    by_id, order = _sorted(ids, 90)
    dy = _matrix(rng.standard_normal((400, 24)), torch.float32)
    dtable, work = torch.empty(60, 24, device=DEV), _bytes(B.adaqp_embedding_backward_workspace_bytes(400, 24))
    B.adaqp_embedding_backward(dy, 24, by_id, order, 1.0, False, dtable, work)
    _check_gradient(dy, np.where(ids < 60, ids, -1), 60, 24, 1.0, dtable)
    far = order.clone()
    far[::5], far[1::5] = -3, 2 ** 31 - 1
    B.adaqp_embedding_backward(dy, 24, by_id, far, 1.0, False, dtable, work)
    far, by_id = far.cpu().numpy(), by_id.cpu().numpy()
    there = (far >= 0) & (far < 400) & (by_id < 60)
    want = np.zeros((60, 24))
    np.add.at(want, by_id[there], _np(dy)[far[there]])
    assert np.allclose(_np(dtable), want, atol=1e-4)


# ---- matrices in 8 bits --------------------------------------------------------------------------------------------------------------------

F8_SHAPES = [(1, 1, None, 0), (3, 5, None, 0), (16, 128, None, 0), (17, 129, 131, 1), (127, 127, None, 0), (128, 256, 256, 0), (129, 602, 608, 0), (70, 602, 640, 0), (300, 301, None, 0), (260, 40, 40, 3),
             (1000, 8, 8, 0), (257, 1024, 1024, 0)]


def _wild(rows, cols, rng):
    """Magnitudes from the bottom of fp32 to its top, zeros, ties, constant blocks, infinities and NaN."""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 21, size=(rows, 1)))
    x[::5] = np.round(x[::5] * 16) / 16
    if rows > 12:
        x[1] = 0.0
        x[2] *= np.exp2(-130.0)
        x[3] = -0.0
        x[4] = rng.choice([-1, 1], cols) * 2.0 ** 128 * (1 - 2.0 ** -24)
        x[6] = rng.standard_normal(cols) * 2.0 ** 125
        x[7] = 448.0
        x[9, cols // 2] = np.inf
        x[11, cols // 3] = np.nan
    return np.clip(x, -3.4028234663852886e38, 3.4028234663852886e38) if rows <= 12 else np.where(np.isfinite(x), np.clip(x, -3.4028234663852886e38, 3.4028234663852886e38), x)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,ld,offset", F8_SHAPES)
def test_f8_quantize_is_the_definition(rows, cols, ld, offset, kind):
    _say("f8 quantize", rows, cols, ld, offset, kind)
    dtype = TYPES[kind]
    xd = _matrix(_wild(rows, cols, np.random.default_rng(rows + cols)), dtype, ld, offset)
    x = _np(xd)
    for blocks in (B.F8_ROWS, B.F8_TILES):
        tiles = blocks == B.F8_TILES
        want, want_t = O.f8_quantize(x, tiles), O.f8_quantize(x.T, tiles)
        for forms in ((True, False), (False, True), (True, True)):
            both = [B.f8_empty(*size, DEV) if form else None for size, form in zip(((rows, cols), (cols, rows)), forms)]
            for packed in both:
                for t in packed or ():
                    t.fill_(0xAA)
            B.adaqp_f8_quantize(xd, cols, blocks, *both)
            for packed, w in zip(both, (want, want_t)):
                if packed is not None:
                    assert np.array_equal(packed[1].cpu().numpy(), w[1]), (blocks, forms)
                    assert np.array_equal(packed[0].cpu().numpy(), w[0]), (blocks, forms)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,ld,offset", F8_SHAPES)
def test_f8_dequantize_is_exact(rows, cols, ld, offset, kind):
    _say("f8 dequantize", rows, cols, ld, offset, kind)
    dtype, rng = TYPES[kind], np.random.default_rng(rows * cols)
    codes, scales = rng.integers(0, 256, (rows, -(-cols // 128) * 128)).astype(np.uint8), rng.integers(0, 256, (-(-cols // 128), -(-rows // 16) * 16)).astype(np.uint8)
    scales[0, 0] = 0
    x, buf = _out(rows, cols, dtype, ld, offset)
    B.adaqp_f8_dequantize((_vec(codes, torch.uint8), _vec(scales, torch.uint8)), cols, x)
    want = torch.from_numpy(O.f8_values(codes, scales, cols)).float().to(dtype)
    assert np.array_equal(_np(x), want.double().numpy(), equal_nan=True)
    _untouched(buf, rows, cols, ld, offset, dtype)


def _f8(values, tiles=False):
    codes, scales = O.f8_quantize(values, tiles)
    return (_vec(codes, torch.uint8), _vec(scales, torch.uint8)), O.f8_values(codes, scales, values.shape[1])


# every tile and the split, edges of each, depths below and across lines, half lines and stages
PRODUCTS = [(1, 1, 1), (5, 3, 7), (32, 32, 128), (33, 31, 129), (7, 300, 602), (32, 1000, 4096), (3, 40, 20_000), (64, 64, 64), (65, 63, 65), (130, 70, 200), (200, 257, 320), (100, 100, 384), (257, 300, 450),
            (256, 300, 5000), (300, 602, 9000), (700, 1100, 256), (1500, 1300, 192), (90, 50, 100_000)]


def _cut_off(a64, b64):
    """Of bf16 outputs of more than 32 rows: the products of eight columns are added to 14 bits of the largest, and each of the seven others loses less than 2^-13 of it."""
    a, b = (torch.from_numpy(np.abs(np.pad(v, ((0, 0), (0, -v.shape[1] % 8))))).to(DEV) for v in (a64, b64))
    total = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=DEV)
    for at in range(0, a.shape[1], 8):
        most = torch.zeros_like(total)
        for k in range(at, at + 8):
            most = torch.maximum(most, torch.outer(a[:, k], b[:, k]))
        total += most
    return 7 * 2.0 ** -13 * total.cpu().numpy()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_f8_matmul(m, n, k, kind):
    _say("f8 matmul", m, n, k, kind)
    dtype, rng = TYPES[kind], np.random.default_rng(m + n + k)
    a, a64 = _f8(rng.standard_normal((m, k)) * np.exp2(rng.integers(-6, 7, size=(m, 1))))
    b, b64 = _f8(rng.standard_normal((n, k)) * np.exp2(rng.integers(-6, 7, size=(n, 1))), tiles=True)
    work = _bytes(B.adaqp_f8_matmul_workspace_bytes(m, n, k))
    work.fill_(0xFF)
    want, terms = a64 @ b64.T, np.abs(a64) @ np.abs(b64).T
    tol = 2 * U * (k / 64 + 16) * terms
    if kind == "bf16" and m > 32:
        tol = tol + _cut_off(a64, b64)
    for ld, offset in ((n, 0), (n + 3, 1), (-(-n // 64) * 64, 0)):
        out, buf = _out(m, n, dtype, ld, offset)
        B.adaqp_f8_matmul(a, b, k, out, work)
        assert np.all(np.abs(_np(out) - want) <= tol + _rounding(np.abs(want) + tol, dtype) + 1e-38)
        _untouched(buf, m, n, ld, offset, dtype)


@pytest.mark.parametrize("m,n,k", [(6000, 5000, 64), (6000, 5000, 640), (8192, 4224, 1600), (8190, 4097, 1700), (40_000, 200, 300), (20_000, 100, 200)])
def test_f8_matmul_of_large_tiles(m, n, k):
    """Against the same values in float64 on the device."""
    _say("f8 matmul large", m, n, k)
    gen = torch.Generator(device=DEV).manual_seed(k)
    a, b = B.f8_empty(m, k, DEV), B.f8_empty(n, k, DEV)
    B.adaqp_f8_quantize(torch.randn(m, k, generator=gen, device=DEV), k, B.F8_ROWS, a, None)
    B.adaqp_f8_quantize(torch.randn(n, k, generator=gen, device=DEV), k, B.F8_TILES, b, None)
    x, y = torch.empty(m, k, device=DEV), torch.empty(n, k, device=DEV)
    B.adaqp_f8_dequantize(a, k, x)
    B.adaqp_f8_dequantize(b, k, y)
    x, y = x.double(), y.double()
    want, terms = x @ y.t(), x.abs() @ y.abs().t()
    for dtype, rounding in ((torch.float32, U), (torch.bfloat16, 2.0 ** -8)):
        out = torch.full((m, n), float("nan"), dtype=dtype, device=DEV)
        B.adaqp_f8_matmul(a, b, k, out, _bytes(B.adaqp_f8_matmul_workspace_bytes(m, n, k)))
        tol = 2 * U * (k / 64 + 16) * terms + (7 * 2.0 ** -13 * terms if dtype == torch.bfloat16 else 0)       # the largest of eight is at most their sum
        assert torch.all((out.double() - want).abs() <= tol + rounding * (want.abs() + tol))


def test_f8_matmul_of_extreme_scales_nan_blocks_and_nothing():
    rng = np.random.default_rng(9)
    for m, n in ((20, 70), (200, 70), (300, 300)):
        _say("f8 matmul extremes", m, n)
        x, y = rng.standard_normal((m, 300)), rng.standard_normal((n, 300))
        x[3] *= 2.0 ** -120
        x[4] *= 2.0 ** 100
        x[5, 200] = np.nan
        y[6, 10] = np.inf
        y[7] = 0.0
        (a, a64), (b, b64) = _f8(x), _f8(y)
        out = torch.full((m, n), SENTINEL, device=DEV)
        work = _bytes(B.adaqp_f8_matmul_workspace_bytes(m, n, 300))
        B.adaqp_f8_matmul(a, b, 300, out, work)
        got, bad = _np(out), np.zeros((m, n), bool)
        bad[5], bad[:, 6] = True, True
        assert np.array_equal(np.isnan(got), bad)
        want, terms = a64 @ b64.T, np.abs(a64) @ np.abs(b64).T
        assert np.all(np.abs(got - want)[~bad] <= (2 * U * 21 * terms + U * np.abs(want))[~bad] + 1e-38)
        B.adaqp_f8_matmul(B.f8_empty(m, 0, DEV), B.f8_empty(n, 0, DEV), 0, out, None)
        assert not out.any()


# ---- log probabilities -------------------------------------------------------------------------------------------------------------------

CLASSES = [(1, 1), (3, 2), (7, 5), (64, 41), (300, 47), (33, 64), (17, 65), (20, 107), (9, 512), (9, 513), (40, 1000), (5, 2048), (5, 2049), (3, 5000), (600, 3001), (2, 8192), (1, 30_000), (3, 65_537),
           (1, 131_072)]


def _logits(rows, classes, rng):
    x = 3 * rng.standard_normal((rows, classes))
    if rows > 2:
        x[1] = 0.25                                  # equal logits
        x[2, rng.integers(classes)] += 40            # one class all but certain
    if rows > 4:
        x[3, rng.random(classes) < 0.7] = -np.inf    # classes that are ruled out
        x[3, classes // 2] = 1.0
        x[4] = -1e4 + 30 * x[4]
    return x


def _prob_tolerances(x, rest):
    """Of rest and entropy.  exp of u = x - max is off by (2 |u| + 4) u (u's own rounding, the product with log2 e, the instruction), relatively; at each of at most classes / 512 + 24 joins a part
    is multiplied by such an exp, of differences whose sum is at most the row's range; additions: classes / 64 + 40 in turn."""
    with np.errstate(invalid="ignore"):
        u = x - x.max(1, keepdims=True)
    e = np.exp(u)
    size = np.where(e > 0, np.abs(u), 0.0)
    span = np.minimum(size.max(1), 104.0)
    n = x.shape[1]
    rel = (n / 64 + 40 + 5 * (n / 512 + 24) + 3 * span) * U
    others, moment = e.sum(1), (size * e).sum(1)
    off = rel * (others - 1) + (U * (2 * size + 4) * e).sum(1) + U
    off_rest = off / others + 2 * U * rest
    off_moment = (rel * moment + (U * (3 * size + 8) * size * e).sum(1)) / others + moment / others * (off / others)
    return off_rest, off_rest + off_moment + 4 * U * (rest + moment / others)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,classes", CLASSES)
def test_logprob_forward_and_backward(rows, classes, kind):
    dtype, rng = TYPES[kind], np.random.default_rng(classes)
    x64 = _logits(rows, classes, rng)
    targets = rng.integers(0, classes, rows)
    if rows > 4:
        targets[0], targets[4] = -1, classes
        targets[2] = int(x64[2].argmax())
    n_top = min(classes, int(rng.integers(1, 33)))
    dlogp, dentropy = rng.standard_normal(rows), rng.standard_normal(rows)
    for ld, offset in ((classes, 0), (classes + 5, 3), (-(-classes // 64) * 64, 0)):
        _say("logprob", rows, classes, n_top, ld, offset, kind)
        xd = _matrix(x64, dtype, ld, offset)
        x = _np(xd)
        logp, top, rest, entropy = O.log_probabilities(x)
        outs = [torch.full((rows + 1,), SENTINEL, device=DEV) for _ in range(2)]
        stats, top_logp = torch.full((rows + 1, 2), SENTINEL, device=DEV), torch.full((rows, n_top), SENTINEL, device=DEV)
        top_class = torch.full((rows, n_top), -9, dtype=torch.int32, device=DEV)
        td, work = _vec(targets, torch.int32), _bytes(B.adaqp_logprob_workspace_bytes(rows, classes, n_top))
        work.fill_(0xFF)
        B.adaqp_logprob_forward(xd, classes, td, outs[0], outs[1], stats, top_logp, top_class, work)
        given = (targets >= 0) & (targets < classes)
        at = np.clip(targets, 0, classes - 1)
        want = np.where(given, logp[np.arange(rows), at], 0.0)
        off_rest, off_entropy = _prob_tolerances(x, rest)
        got = _np(outs[0])
        with np.errstate(invalid="ignore"):
            u = np.where(given, x[np.arange(rows), at] - top, 0.0)
            close = np.abs(got[:rows] - want) <= off_rest + U * np.abs(u) + U * np.abs(want)
        assert np.all(close | (got[:rows] == want))
        assert np.all(np.abs(_np(outs[1])[:rows] - entropy) <= off_entropy)
        assert np.array_equal(_np(stats)[:rows, 0], top) and np.all(np.abs(_np(stats)[:rows, 1] - rest) <= off_rest)
        assert outs[0][rows] == SENTINEL and outs[1][rows] == SENTINEL and torch.all(stats[rows] == SENTINEL)
        classes_want = O.largest(x, n_top)
        assert np.array_equal(top_class.cpu().numpy(), classes_want)
        with np.errstate(invalid="ignore"):
            u = np.take_along_axis(x, classes_want, 1) - top[:, None]
            tops = u - rest[:, None]
            close = np.abs(_np(top_logp) - tops) <= off_rest[:, None] + U * (np.abs(u) + np.abs(tops))
        assert np.all(close | (_np(top_logp) == tops))
        # without some of the outputs: the same bits
        only = torch.empty(rows, device=DEV)
        B.adaqp_logprob_forward(xd, classes, None, None, only, None, workspace=work)
        assert torch.equal(only, outs[1][:rows])
        B.adaqp_logprob_forward(xd, classes, td, only, workspace=work)
        assert torch.equal(only, outs[0][:rows])
        # the gradient, by the statistics that the call is given
        given_stats, given_entropy = _np(stats)[:rows], _np(outs[1])[:rows]
        gp, gh = _vec(dlogp), _vec(dentropy)
        dlogp64, dentropy64 = _np(gp), _np(gh)
        for with_dlogp, with_dentropy, scale in ((True, True, 0.7), (False, False, -1.0 / rows), (False, True, 3.0)):
            d, buf = _out(rows, classes, dtype, ld, offset)
            B.adaqp_logprob_backward(xd, classes, td, stats, outs[1], gp if with_dlogp else None, gh if with_dentropy else None, scale, d)
            gl, ge = dlogp64 if with_dlogp else np.ones(rows), dentropy64 if with_dentropy else np.zeros(rows)
            scale32 = float(np.float32(scale))
            want = O.logprob_gradient(x, targets, given_stats[:, 0], given_stats[:, 1], given_entropy, gl, ge, scale32)
            with np.errstate(invalid="ignore"):
                u = np.abs(x - given_stats[:, :1])
                lp = np.minimum(u + given_stats[:, 1:], 300.0)
                p = np.exp(-(u + given_stats[:, 1:]))
            # exp(logp) is off by |u| + 3 |logp| + 4 roundings; of what it is multiplied with each rounds once
            rel = U * (np.minimum(u, 300.0) + 3 * lp + 8)
            H = np.abs(given_entropy)[:, None]
            one = np.zeros(p.shape)
            one[np.nonzero(given)[0], targets[given]] = 1.0
            tol = abs(scale32) * (np.where(given, np.abs(gl), 0.0)[:, None] * (p * rel + 4 * U * one) + np.abs(ge)[:, None] * p * ((lp + H) * (rel + 4 * U) + U * (np.minimum(u, 300.0) + 2 * lp + H))) + 4 * U * np.abs(want)
            # a p below 2^-126 = 1.2e-38 is no normal number and may be taken for zero: what is lost is what it was to be multiplied with times that (p = 1.2e-39, |logp| = 90, scale 3: 1.5e-37)
            tol = tol + 2.0 ** -126 * (1 + abs(scale32) * (np.abs(gl)[:, None] + np.abs(ge)[:, None] * (lp + H)))
            assert np.all(np.abs(_np(d) - want) <= tol + _rounding(np.abs(want) + tol, dtype))
            _untouched(buf, rows, classes, ld, offset, dtype)
    again = xd.clone() if xd.is_contiguous() else xd
    B.adaqp_logprob_backward(again, classes, td, stats, outs[1], None, gh, 3.0, again)           # in place
    assert torch.equal(again, d)


@pytest.mark.parametrize("classes", [5, 41, 700, 3000, 20_000])
def test_logprob_of_rows_that_are_empty_or_not_finite(classes):
    _say("logprob edges", classes)
    rng = np.random.default_rng(classes)
    x = rng.standard_normal((7, classes))
    x[1] = -np.inf
    x[2, classes // 2] = np.nan
    x[3, classes - 1] = np.inf
    x[4] = -np.inf
    x[4, 2] = -3.0                                   # one class is left
    x[5] = np.nan
    xd = _matrix(x, torch.float32)
    targets = np.array([0, 1, 2, 3, 2, 0, -1])
    td, n_top = _vec(targets, torch.int32), min(4, classes)
    logp, entropy, stats, top_logp = (torch.full(s, SENTINEL, device=DEV) for s in ((7,), (7,), (7, 2), (7, n_top)))
    top_class = torch.empty(7, n_top, dtype=torch.int32, device=DEV)
    B.adaqp_logprob_forward(xd, classes, td, logp, entropy, stats, top_logp, top_class, _bytes(B.adaqp_logprob_workspace_bytes(7, classes, n_top)))
    logp, entropy, top_logp = _np(logp), _np(entropy), _np(top_logp)
    assert logp[1] == -np.inf and entropy[1] == 0 and np.all(top_logp[1] == -np.inf) and stats[1].tolist() == [-np.inf, 0]
    for bad in (2, 3, 5):
        assert np.isnan(logp[bad]) and np.isnan(entropy[bad]) and np.isnan(top_logp[bad]).all() and torch.isnan(stats[bad, 1])
    assert logp[4] == 0 and entropy[4] == 0 and top_logp[4, 0] == 0 and np.all(top_logp[4, 1:] == -np.inf)
    assert logp[6] == 0 and np.isfinite(logp[0])
    assert np.array_equal(top_class.cpu().numpy(), O.largest(x, n_top))
    d = torch.full((7, classes), SENTINEL, device=DEV)
    B.adaqp_logprob_backward(xd, classes, td, stats, None, None, None, 1.0, d)
    d = _np(d)
    assert not d[1].any() and not d[6].any() and np.isnan(d[[2, 3, 5]]).all() and np.isfinite(d[[0, 4]]).all() and not d[4].any()
    d = torch.full((7, classes), SENTINEL, device=DEV)
    B.adaqp_logprob_backward(xd, classes, None, stats, _vec(entropy), None, torch.ones(7, device=DEV), 1.0, d)
    d = _np(d)
    assert not d[1].any() and not d[4].any() and np.isnan(d[[2, 3, 5]]).all() and np.isfinite(d[[0, 6]]).all() and d[6].any()


def test_logprob_keeps_the_digits_of_what_is_all_but_certain():
    """A class with the probability 1 - 1e-9: its log probability, the entropy and 1 - p have the digits of fp32."""
    x = np.zeros((2, 300))
    x[:, 1:] = -np.log(299e9)
    xd = _matrix(x, torch.float32)
    logp, entropy, stats = torch.empty(2, device=DEV), torch.empty(2, device=DEV), torch.empty(2, 2, device=DEV)
    td = _vec([0, 0], torch.int32)
    B.adaqp_logprob_forward(xd, 300, td, logp, entropy, stats)
    want, _, _, want_entropy = O.log_probabilities(_np(xd))
    assert np.all(np.abs(_np(logp) - want[:, 0]) <= 1e-5 * np.abs(want[:, 0])) and np.all(np.abs(_np(entropy) - want_entropy) <= 1e-5 * want_entropy)
    d = torch.empty(2, 300, device=DEV)
    B.adaqp_logprob_backward(xd, 300, td, stats, None, None, None, 1.0, d)
    assert np.all(np.abs(_np(d)[:, 0] + np.expm1(want[:, 0])) <= 1e-5 * np.abs(want[:, 0]))


@pytest.mark.parametrize("classes,n_top", [(41, 5), (600, 32), (5000, 20), (40_000, 32)])
def test_largest_of_rows_with_many_equal_and_in_every_order(classes, n_top):
    _say("largest", classes, n_top)
    rng = np.random.default_rng(classes)
    up = np.arange(classes, dtype=np.float64) / 64
    x = np.stack([up, up[::-1], np.zeros(classes), rng.integers(0, 3, classes), np.where(rng.random(classes) < 0.5, 0.0, -0.0), rng.integers(0, classes // 8, classes), -up * 1e30])
    x[6, 5:] = -np.inf
    for dtype in TYPES.values():
        xd = _matrix(x, dtype, classes + 1, 1)
        top_logp, top_class = torch.empty(7, n_top, device=DEV), torch.empty(7, n_top, dtype=torch.int32, device=DEV)
        B.adaqp_logprob_forward(xd, classes, None, None, None, None, top_logp, top_class, _bytes(B.adaqp_logprob_workspace_bytes(7, classes, n_top)))
        assert np.array_equal(top_class.cpu().numpy(), O.largest(_np(xd), n_top))


# ---- streams and graphs ------------------------------------------------------------------------------------------------------------------

def _program(gen):
    """All calls on buffers of their own; returns (inputs, what runs them, outputs)."""
    n, entries, dim, classes = 700, 90, 72, 41
    ids = torch.randint(-1, entries, (n,), generator=gen, device=DEV, dtype=torch.int32)
    table, w = torch.randn(entries, dim, generator=gen, device=DEV), torch.randn(classes, dim, generator=gen, device=DEV)
    targets = torch.randint(-1, classes, (n,), generator=gen, device=DEV, dtype=torch.int32)
    counter = torch.zeros(1, dtype=torch.int64, device=DEV)
    e = lambda *s, **k: torch.empty(*s, device=DEV, **k)  # noqa: E731
    h, d, z, logp, entropy, stats, dz, dh, dd, dw, dtable = e(n, dim), e(n, dim), e(n, classes), e(n), e(n), e(n, 2), e(n, classes), e(n, dim), e(n, dim), e(classes, dim), e(entries, dim)
    by_id, order = e(n, dtype=torch.int32), e(n, dtype=torch.int32)
    top, top_class = e(n, 3), e(n, 3, dtype=torch.int32)
    h8, ht8, w8, wt8, dz8, dzt8 = (B.f8_empty(*s, DEV) for s in ((n, dim), (dim, n), (classes, dim), (dim, classes), (n, classes), (classes, n)))
    work = _bytes(max(B.adaqp_embedding_sort_workspace_bytes(n, entries), B.adaqp_embedding_backward_workspace_bytes(n, dim), B.adaqp_f8_matmul_workspace_bytes(n, classes, dim),
                      B.adaqp_f8_matmul_workspace_bytes(n, dim, classes), B.adaqp_f8_matmul_workspace_bytes(classes, dim, n), B.adaqp_logprob_workspace_bytes(n, classes, 3)))

    def run(stream=None):
        B.adaqp_embedding_forward(table, dim, ids, 2.0, h, stream=stream)
        B.adaqp_dropout(h, dim, 0.3, 11, d, counter=counter, stream=stream)
        B.adaqp_f8_quantize(d, dim, B.F8_ROWS, h8, ht8, stream=stream)
        B.adaqp_f8_quantize(w, dim, B.F8_TILES, w8, wt8, stream=stream)
        B.adaqp_f8_matmul(h8, w8, dim, z, work, stream=stream)
        B.adaqp_logprob_forward(z, classes, targets, logp, entropy, stats, top, top_class, work, stream=stream)
        B.adaqp_logprob_backward(z, classes, targets, stats, entropy, None, None, -1.0 / n, dz, stream=stream)
        B.adaqp_f8_quantize(dz, classes, B.F8_ROWS, dz8, dzt8, stream=stream)
        B.adaqp_f8_matmul(dz8, wt8, classes, dd, work, stream=stream)
        B.adaqp_f8_matmul(dzt8, ht8, n, dw, work, stream=stream)
        B.adaqp_dropout(dd, dim, 0.3, 11, dh, counter=counter, stream=stream)
        B.adaqp_embedding_sort(ids, entries, by_id, order, work, stream=stream)
        B.adaqp_embedding_backward(dh, dim, by_id, order, 2.0, False, dtable, work, stream=stream)
    return dict(ids=ids, table=table, w=w, targets=targets, counter=counter), run, [logp, entropy, top, top_class, dw, dtable]


def test_a_step_of_all_of_them_has_the_slopes_of_its_loss():
    """The gradients that the calls hand on from one to the next, against the loss's own definition with the operands as they were rounded: product of held values, straight through the
    rounding."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    inputs, run, (logp, entropy, top, top_class, dw, dtable) = _program(gen)
    run()
    n, entries, dim, classes = 700, 90, 72, 41
    ids, targets = inputs["ids"].cpu().numpy(), inputs["targets"].cpu().numpy()
    keep, factor = O.dropped(n, dim, 0.3, 11)
    h = O.embedding(_np(inputs["table"]), ids, 2.0).astype(np.float32)
    d = np.where(keep, h * np.float32(factor), np.float32(0)).astype(np.float64)
    held = lambda v, tiles=False: O.f8_values(*O.f8_quantize(v, tiles), v.shape[1])  # noqa: E731
    d8, w8 = held(d), held(_np(inputs["w"]), True)
    z = d8 @ w8.T
    lp, most, rest, H = O.log_probabilities(z)
    given = targets >= 0
    # a logit is off by an fp32 sum's rounding, a log probability by twice that, the entropy by that times the range of the logits, which is below 40
    off = 2 * U * (dim / 64 + 16) * (np.abs(d8) @ np.abs(w8).T).max() + 1e-6
    assert np.abs(_np(logp) - np.where(given, lp[np.arange(n), np.maximum(targets, 0)], 0)).max() <= 2 * off and np.abs(_np(entropy) - H).max() <= 40 * off
    dz = O.logprob_gradient(z, targets, most, rest, H, np.ones(n), np.zeros(n), -1.0 / n)
    # dz differs from the calls' by roundings, relatively by 1e-4 at most, and where that crosses a border of two codes by a step, 2^-3 of it: in at most a share of 1e-4 * 2^4 of the elements.  Their
    # squares add up to 1.6e-3 * 2^-6 of all: a root mean square of 5e-3 of dz's
    want_w, want_d = held(dz.T) @ held(d.T).T, np.where(keep, held(dz) @ w8 * factor, 0)
    want_t = O.embedding_gradient(want_d, ids, entries, 2.0)
    for got, want in ((dw, want_w), (dtable, want_t)):
        assert np.sqrt(((_np(got) - want) ** 2).mean()) <= 5e-3 * np.sqrt((want ** 2).mean())


def test_calls_follow_their_stream():
    gen = torch.Generator(device=DEV).manual_seed(1)
    inputs, run, outputs = _program(gen)
    run()
    want = [t.clone() for t in outputs]
    torch.cuda.synchronize()
    for how in ("argument", "current"):
        for t in outputs:
            t.fill_(7)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        if how == "argument":
            run(stream)
        else:
            with torch.cuda.stream(stream):
                run()
        stream.synchronize()
        for got, w in zip(outputs, want):
            assert torch.equal(got, w)


def test_calls_can_be_captured():
    """One graph of all calls, replayed on inputs that change, between the program's own work: every replay as the calls themselves, the counter's numbers among them."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    inputs, run, outputs = _program(gen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    seen = []
    for step in range(4):
        _say("replay", step)
        inputs["table"].copy_(torch.randn(90, 72, generator=gen, device=DEV))
        inputs["ids"].copy_(torch.randint(-1, 90, (700,), generator=gen, device=DEV, dtype=torch.int32))
        inputs["counter"].fill_(step // 2)
        graph.replay()
        got = [t.clone() for t in outputs]
        torch.cuda.synchronize()
        for t in outputs:
            t.fill_(3)
        run()
        for g, t in zip(got, outputs):
            assert torch.equal(g, t)
        seen.append(got[0])
    assert not torch.equal(seen[0], seen[3])
