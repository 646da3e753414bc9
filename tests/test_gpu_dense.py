"""The dense operators on the GPU against their float64 definitions (oracle/dense.py).

u = 2^-24.  Tolerances follow from the number of roundings: a sum of t terms taken by lanes in turn and then joined is off by at most (t / lanes + 16) u of
the sum of the terms' magnitudes; each further operation adds u.  bf16 outputs (7 stored bits) add half a unit in their last place, at most 2^-8 of the value."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dense as D                                        # noqa: E402
from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
SENTINEL = -77.0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def _say(*what):
    print(*what, flush=True)
    sys.stdout.flush()


def _matrix(values, dtype, ld=None, offset=0, padding=float("nan")):
    """`values` as a device matrix of pitch ld whose first element lies `offset` elements behind a 128-byte line; what is behind the columns holds `padding`."""
    rows, cols = values.shape
    ld = ld or cols
    buf = torch.full((rows * ld + offset + 256,), padding, dtype=dtype, device=DEV)
    m = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.from_numpy(np.asarray(values, dtype=np.float64)).to(dtype))
    return m


def _out(rows, cols, dtype, ld=None, offset=0):
    buf = torch.full((rows * (ld or cols) + offset + 256,), SENTINEL, dtype=dtype, device=DEV)
    return buf[offset:offset + rows * (ld or cols)].view(rows, ld or cols)[:, :cols], buf


def _np(t):
    return t.double().cpu().numpy()


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def _rounding(values, dtype):
    return (2.0 ** -8 if dtype == torch.bfloat16 else U) * np.abs(values)


def _untouched(buf, m, rows, cols, ld, offset, dtype):
    """Only the matrix's columns were written or, with rows of whole lines, its lines, the padding with zeros."""
    b = _np(buf)
    assert np.all(b[:offset] == SENTINEL) and np.all(b[offset + rows * ld:] == SENTINEL)
    line = 128 // dtype.itemsize
    behind = b[offset:offset + rows * ld].reshape(rows, ld)[:, cols:]
    if offset == 0 and ld % line == 0:
        written = -(-cols // line) * line - cols
        assert np.all(behind[:, :written] == 0) and np.all(behind[:, written:] == SENTINEL)
    else:
        assert np.all(behind == SENTINEL)


# ---- layer norm ------------------------------------------------------------------------------------------------------------------------------------

SHAPES = [  # rows, dim, ld, offset
    (1, 1, None, 0), (1, 128, None, 0), (3, 5, None, 0), (17, 16, None, 0), (33, 31, 33, 1), (130, 64, 64, 0), (1000, 256, 256, 0), (64, 256, 300, 0),
    (50, 301, None, 0), (70, 602, 608, 0), (70, 602, 640, 0), (70, 602, None, 0), (21, 604, 604, 4), (40, 514, 520, 2), (9, 1023, None, 0), (11, 1500, 1500, 0),
    (12, 2047, None, 0), (12, 2048, 2048, 0), (7, 2049, 2112, 0), (5, 4097, None, 0), (5, 8192, 8192, 0), (3, 8200, None, 0), (2, 20_001, 20_032, 0),
    (5000, 48, 64, 0), (2500, 100, 100, 0),
]


def _norm_values(rows, dim, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, dim)) * np.exp2(rng.integers(-8, 9, size=(rows, 1))) + rng.standard_normal((rows, 1)) * 3
    if rows > 2:
        x[1] = 0.375                                 # a constant row
        x[2] = 0.0
    return x, 1 + 0.3 * rng.standard_normal(dim), rng.standard_normal(dim), rng.standard_normal((rows, dim))


def _vec(v):
    return torch.from_numpy(np.asarray(v, dtype=np.float32)).to(DEV)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,dim,ld,offset", SHAPES)
def test_layernorm_forward(rows, dim, ld, offset, kind):
    _say("layernorm forward", rows, dim, ld, offset, kind)
    dtype = TYPES[kind]
    x, gamma, beta, _ = _norm_values(rows, dim, dim)
    xd = _matrix(x, dtype, ld, offset)
    gd, bd = _vec(gamma), _vec(beta)
    eps = 1e-5
    y, buf = _out(rows, dim, dtype, ld, offset)
    stats = torch.full((rows, 2), SENTINEL, device=DEV)
    B.adaqp_layernorm_forward(xd, dim, gd, bd, eps, y, stats)
    x = _np(xd)
    want, mean, rstd = D.layernorm(x, _np(gd), _np(bd), np.float32(eps))
    k = dim / 64 + 48
    off_mean = k * U * np.abs(x).mean(1)
    h = (x - mean[:, None]) * rstd[:, None]
    # d = x - mean is off by off_mean + u |d|; rstd by half the relative error of the mean square, where the error of the mean enters as its square over the variance
    rel = (k + 8) * U + 0.5 * (off_mean * rstd) ** 2
    tol = np.abs(_np(gd)) * ((off_mean * rstd)[:, None] * (1 + rel[:, None]) + np.abs(h) * rel[:, None]) + 4 * U * (np.abs(h * _np(gd)) + np.abs(_np(bd)))
    got = _np(y)
    assert np.all(np.abs(got - want) <= tol + _rounding(np.abs(want) + tol, dtype) + 1e-38)
    assert np.all(np.abs(_np(stats)[:, 0] - mean) <= off_mean + 1e-38) and np.all(np.abs(_np(stats)[:, 1] - rstd) <= rel * rstd)
    _untouched(buf, y, rows, dim, ld or dim, offset, dtype)
    again, _ = _out(rows, dim, dtype, ld, offset)
    B.adaqp_layernorm_forward(xd, dim, gd, bd, eps, again)
    assert torch.equal(again, y)
    B.adaqp_layernorm_forward(xd, dim, gd, bd, eps, xd)              # in place
    assert torch.equal(xd, y)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,dim,ld,offset", SHAPES)
def test_layernorm_backward(rows, dim, ld, offset, kind):
    _say("layernorm backward", rows, dim, ld, offset, kind)
    dtype = TYPES[kind]
    x, gamma, _, dy = _norm_values(rows, dim, dim + 1)
    xd, dyd, gd = _matrix(x, dtype, ld, offset), _matrix(dy, dtype, ld, offset), _vec(gamma)
    x, dy, gamma = _np(xd), _np(dyd), _np(gd)
    _, mean, rstd = D.layernorm(x, 1.0, 0.0, 1e-5)
    stats = torch.from_numpy(np.stack([mean, rstd], 1)).float().to(DEV)
    mean, rstd = _np(stats).T
    dx, buf = _out(rows, dim, dtype, ld, offset)
    dgamma, dbeta = torch.full((dim,), SENTINEL, device=DEV), torch.full((dim,), SENTINEL, device=DEV)
    work = _bytes(B.adaqp_layernorm_workspace_bytes(rows, dim))
    B.adaqp_layernorm_backward(xd, dyd, dim, stats, gd, dx, dgamma, dbeta, work)
    want, want_gamma, want_beta = D.layernorm_backward(x, dy, mean, rstd, gamma)
    h, g = (x - mean[:, None]) * rstd[:, None], dy * gamma
    k = dim / 64 + 56
    tol = rstd[:, None] * U * (8 * np.abs(g) + k * np.abs(g).mean(1)[:, None] + (k + 8) * np.abs(h) * np.abs(g * h).mean(1)[:, None])
    assert np.all(np.abs(_np(dx) - want) <= tol + _rounding(np.abs(want) + tol, dtype) + 1e-38)
    many = rows / 64 + 64
    assert np.all(np.abs(_np(dgamma) - want_gamma) <= (many + 4) * U * np.abs(dy * h).sum(0) + 1e-38)
    assert np.all(np.abs(_np(dbeta) - want_beta) <= many * U * np.abs(dy).sum(0) + 1e-38)
    _untouched(buf, dx, rows, dim, ld or dim, offset, dtype)
    # without the input's gradient, without the parameters', in place of dy: the same bits
    only = [torch.empty_like(dgamma), torch.empty_like(dbeta)]
    B.adaqp_layernorm_backward(xd, dyd, dim, stats, gd, None, *only, work)
    assert torch.equal(only[0], dgamma) and torch.equal(only[1], dbeta)
    B.adaqp_layernorm_backward(xd, dyd, dim, stats, gd, dyd, None, None, None)
    assert torch.equal(dyd, dx)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("dim", [1, 20, 31, 33, 64, 100, 300, 602, 1000, 2100])
def test_layernorm_of_matrices_that_lie_differently(dim, kind):
    """One with whole lines, one that begins anywhere: the definition's values (tolerances as above), and padding only where it is."""
    _say("layernorm mixed", dim, kind)
    dtype, rows = TYPES[kind], 37
    x, gamma, beta, dy = _norm_values(rows, dim, dim)
    padded = -(-dim // 64) * 64
    gd, bd = _vec(gamma), _vec(beta)
    x, dy = _np(_matrix(x, dtype)), _np(_matrix(dy, dtype))
    y64, mean, rstd = D.layernorm(x, _np(gd), _np(bd), np.float32(1e-5))
    stats = torch.from_numpy(np.stack([mean, rstd], 1)).float().to(DEV)
    k = dim / 64 + 48
    off_mean = k * U * np.abs(x).mean(1)
    h = (x - mean[:, None]) * rstd[:, None]
    rel = (k + 8) * U + 0.5 * (off_mean * rstd) ** 2
    tol_y = np.abs(_np(gd)) * ((off_mean * rstd)[:, None] * (1 + rel[:, None]) + np.abs(h) * rel[:, None]) + 4 * U * (np.abs(h * _np(gd)) + np.abs(_np(bd)))
    mean, rstd = _np(stats).T
    dx64, dgamma64, dbeta64 = D.layernorm_backward(x, dy, mean, rstd, _np(gd))
    h, g = (x - mean[:, None]) * rstd[:, None], dy * _np(gd)
    k = dim / 64 + 56
    tol_dx = rstd[:, None] * U * (8 * np.abs(g) + k * np.abs(g).mean(1)[:, None] + (k + 8) * np.abs(h) * np.abs(g * h).mean(1)[:, None])
    many = rows / 64 + 64
    work = _bytes(B.adaqp_layernorm_workspace_bytes(rows, dim))
    for ld_in, at_in, ld_out, at_out in ((padded, 0, dim, 0), (dim + 3, 1, padded, 0), (dim, 0, padded, 0), (padded, 0, dim + 1, 1)):
        xd = _matrix(x, dtype, ld_in, at_in)
        y, buf = _out(rows, dim, dtype, ld_out, at_out)
        B.adaqp_layernorm_forward(xd, dim, gd, bd, 1e-5, y)
        assert np.all(np.abs(_np(y) - y64) <= tol_y + _rounding(np.abs(y64) + tol_y, dtype) + 1e-38)
        _untouched(buf, y, rows, dim, ld_out, at_out, dtype)
        dx, buf = _out(rows, dim, dtype, ld_out, at_out)
        dgamma, dbeta = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
        B.adaqp_layernorm_backward(xd, _matrix(dy, dtype), dim, stats, gd, dx, dgamma, dbeta, work)
        assert np.all(np.abs(_np(dx) - dx64) <= tol_dx + _rounding(np.abs(dx64) + tol_dx, dtype) + 1e-38)
        assert np.all(np.abs(_np(dgamma) - dgamma64) <= (many + 4) * U * np.abs(dy * h).sum(0) + 1e-38)
        assert np.all(np.abs(_np(dbeta) - dbeta64) <= many * U * np.abs(dy).sum(0) + 1e-38)
        _untouched(buf, dx, rows, dim, ld_out, at_out, dtype)


def test_layernorm_without_parameters_and_rows():
    x = _matrix(np.random.default_rng(0).standard_normal((4, 32)), torch.float32)
    y, plain = torch.empty_like(x), torch.empty_like(x)
    B.adaqp_layernorm_forward(x, 32, None, None, 1e-5, y)
    B.adaqp_layernorm_forward(x, 32, torch.ones(32, device=DEV), torch.zeros(32, device=DEV), 1e-5, plain)
    assert torch.equal(y, plain)
    dgamma, dbeta = torch.full((32,), SENTINEL, device=DEV), torch.full((32,), SENTINEL, device=DEV)
    none = torch.empty(0, 32, device=DEV)
    B.adaqp_layernorm_backward(none, none, 32, torch.empty(0, 2, device=DEV), None, none, dgamma, dbeta, None)
    assert not dgamma.any() and not dbeta.any()
    B.adaqp_layernorm_forward(none, 32, None, None, 1e-5, none)


def test_layernorm_keeps_what_is_not_finite_in_its_row():
    x = np.random.default_rng(0).standard_normal((6, 70))
    x[1, 3], x[4, 69] = np.inf, np.nan
    xd = _matrix(x, torch.float32)
    y, stats = torch.empty_like(xd), torch.empty(6, 2, device=DEV)
    B.adaqp_layernorm_forward(xd, 70, None, None, 1e-5, y, stats)
    bad = np.isnan(_np(y))
    assert bad[[1, 4]].all() and not bad[[0, 2, 3, 5]].any()
    dx = torch.empty_like(xd)
    B.adaqp_layernorm_backward(xd, torch.ones_like(xd), 70, stats, None, dx, None, None, None)
    bad = np.isnan(_np(dx))
    assert bad[[1, 4]].all() and not bad[[0, 2, 3, 5]].any()


def test_layernorm_gradients_are_differences():
    """d/dt of sum(dy * y) along random directions of x, gamma and beta, from the definition in 64 bits, against the gradients of the GPU."""
    rng = np.random.default_rng(5)
    rows, dim, eps, t = 20, 37, 1e-5, 1e-5
    x, dy, gamma, beta = rng.standard_normal((rows, dim)), rng.standard_normal((rows, dim)), rng.standard_normal(dim), rng.standard_normal(dim)
    x, dy, gamma, beta = (v.astype(np.float32).astype(np.float64) for v in (x, dy, gamma, beta))
    xd, dyd, y, stats = _matrix(x, torch.float32), _matrix(dy, torch.float32), torch.empty(rows, dim, device=DEV), torch.empty(rows, 2, device=DEV)
    B.adaqp_layernorm_forward(xd, dim, _vec(gamma), _vec(beta), eps, y, stats)
    dx, dgamma, dbeta = torch.empty_like(xd), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    B.adaqp_layernorm_backward(xd, dyd, dim, stats, _vec(gamma), dx, dgamma, dbeta, _bytes(B.adaqp_layernorm_workspace_bytes(rows, dim)))

    def loss(x, gamma, beta):
        return (dy * D.layernorm(x, gamma, beta, eps)[0]).sum()
    for _ in range(5):
        vx, vg, vb = rng.standard_normal((rows, dim)), rng.standard_normal(dim), rng.standard_normal(dim)
        slope = (loss(x + t * vx, gamma + t * vg, beta + t * vb) - loss(x - t * vx, gamma - t * vg, beta - t * vb)) / (2 * t)
        got = (_np(dx) * vx).sum() + (_np(dgamma) * vg).sum() + (_np(dbeta) * vb).sum()
        size = np.abs(_np(dx) * vx).sum() + np.abs(_np(dgamma) * vg).sum() + np.abs(_np(dbeta) * vb).sum()
        assert abs(got - slope) <= 1e-5 * size


# ---- MX matrices -------------------------------------------------------------------------------------------------------------------------------------

MX_SHAPES = [(1, 1, None, 0), (1, 32, None, 0), (5, 31, None, 0), (33, 33, 40, 0), (128, 128, None, 0), (127, 129, None, 0), (300, 602, None, 0),
             (130, 602, 608, 0), (64, 300, 304, 4), (257, 256, None, 1), (1000, 70, 72, 0), (3, 1000, None, 0), (129, 64, 66, 2)]


def _mx_values(rows, cols, seed):
    """Magnitudes over many powers of two; zeros, whole blocks of them, ties, subnormals, and blocks with an infinity or NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, size=(rows, cols)))
    x[rng.random((rows, cols)) < 0.1] = 0.0
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 4.0, -0.25, -5.0, -0.0])
    put = rng.random((rows, cols)) < 0.2
    x[put] = grid[rng.integers(0, len(grid), size=int(put.sum()))]
    if rows > 4 and cols > 4:
        x[1, :] = 0.0
        x[2, :] *= 2.0 ** -130
        x[3, :] *= 2.0 ** 100
        x[4, 2], x[0, cols - 1] = np.inf, np.nan
    return x


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("seed", [None, 0x123456789ABCDEF])
@pytest.mark.parametrize("rows,cols,ld,offset", MX_SHAPES)
def test_mx4_quantize_is_the_definition(rows, cols, ld, offset, seed, kind):
    _say("mx4 quantize", rows, cols, ld, offset, seed, kind)
    xd = _matrix(_mx_values(rows, cols, cols), TYPES[kind], ld, offset)
    x = _np(xd)
    want, want_t = D.mx4_quantize(x, seed), D.mx4_quantize(x.T, None if seed is None else seed + 1)
    rounding = B.MX4_NEAREST if seed is None else B.MX4_STOCHASTIC
    for rows_too in (True, False):
        for columns_too in (True, False):
            packed = tuple(t.fill_(0xAB) for t in B.mx4_empty(rows, cols, DEV)) if rows_too else None
            packed_t = tuple(t.fill_(0xAB) for t in B.mx4_empty(cols, rows, DEV)) if columns_too else None
            B.adaqp_mx4_quantize(xd, cols, rounding, seed or 0, packed, packed_t)
            for got, expected in ((packed, want), (packed_t, want_t)):
                if got is not None:
                    assert np.array_equal(got[1].cpu().numpy(), expected[1])
                    assert np.array_equal(got[0].cpu().numpy(), expected[0])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,ld,offset", MX_SHAPES + [(20, 602, 640, 0), (20, 128, 192, 0)])
def test_mx4_dequantize_is_exact(rows, cols, ld, offset, kind):
    _say("mx4 dequantize", rows, cols, ld, offset, kind)
    dtype = TYPES[kind]
    rng = np.random.default_rng(rows)
    codes, scales = B.mx4_empty(rows, cols, "cpu")
    codes = rng.integers(0, 256, size=tuple(codes.shape)).astype(np.uint8)
    scales = rng.integers(0, 253, size=tuple(scales.shape)).astype(np.uint8)
    scales[0, 0, 0] = 255
    scales[-1, -1] = 0
    out, buf = _out(rows, cols, dtype, ld, offset)
    B.adaqp_mx4_dequantize((torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)), cols, out)
    want = D.mx4_values(codes, scales, cols)
    assert np.array_equal(_np(out), want, equal_nan=True)
    _untouched(buf, out, rows, cols, ld or cols, offset, dtype)


PRODUCTS = [(1, 1, 1), (1, 33, 31), (5, 64, 128), (31, 7, 129), (64, 64, 256), (65, 63, 300), (128, 128, 512), (129, 257, 602), (300, 41, 602), (1, 1000, 4096),
            (17, 300, 2000), (2, 2, 60_000), (256, 300, 30_000), (1000, 520, 96), (2100, 2050, 384), (40_000, 16, 40), (16, 40_000, 40), (33, 65, 2049)]


def _mx_random(rows, cols, seed, spread=2):
    x = np.random.default_rng(seed).standard_normal((rows, cols)) * np.exp2(np.random.default_rng(seed + 1).integers(-spread, spread + 1, size=(rows, cols)))
    codes, scales = D.mx4_quantize(x)
    return (torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)), D.mx4_values(codes, scales, cols)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_mx4_matmul(m, n, k, kind):
    _say("mx4 matmul", m, n, k, kind)
    dtype = TYPES[kind]
    a, av = _mx_random(m, k, 3 * m + k)
    b, bv = _mx_random(n, k, 5 * n + k)
    work = _bytes(B.adaqp_mx4_matmul_workspace_bytes(m, n, k)).fill_(0xFF)
    want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
    for ld in {n, -(-n // 64) * 64, n + 3}:
        out, buf = _out(m, n, dtype, ld)
        B.adaqp_mx4_matmul(a, b, k, out, work)
        tol = 2 * U * (k / 64 + 16) * size
        assert np.all(np.abs(_np(out) - want) <= tol + _rounding(np.abs(want) + tol, dtype))
        _untouched(buf, out, m, n, ld, 0, dtype)
    again = torch.empty(m, n, dtype=dtype, device=DEV)
    B.adaqp_mx4_matmul(a, b, k, again, work)
    assert torch.equal(again, out)


@pytest.mark.parametrize("m,n,k", [(4200, 2040, 1600), (8200, 4090, 3200), (256, 602, 9000), (100, 90, 20_000), (30, 20, 70_000), (600, 30_000, 700)])
def test_mx4_matmul_of_every_tile(m, n, k):
    """The sizes that the larger tiles and the cut sums are for; products by torch in float64 of the values."""
    _say("mx4 matmul tiles", m, n, k)
    gen = torch.Generator(device=DEV).manual_seed(m)
    packed, values = [], []
    for rows in (m, n):
        codes, scales = B.mx4_empty(rows, k, DEV)
        packed.append((codes.random_(0, 256, generator=gen), scales.random_(125, 130, generator=gen)))
        if k % 128:
            codes[:, k // 2 + k % 2:].zero_()
            if k % 2:
                codes[:, k // 2] &= 15
        values.append(torch.from_numpy(D.mx4_values(codes.cpu().numpy(), scales.cpu().numpy(), k)).to(DEV))
    out = torch.empty(m, n, device=DEV)
    B.adaqp_mx4_matmul(*packed, k, out, _bytes(B.adaqp_mx4_matmul_workspace_bytes(m, n, k)).fill_(0xFF))
    want, size = values[0] @ values[1].t(), values[0].abs() @ values[1].abs().t()
    assert bool(((out.double() - want).abs() <= 2 * U * (k / 64 + 16) * size).all())


@pytest.mark.parametrize("m,n,k", [(9000, 300, 40), (9001, 301, 500), (8999, 260, 640), (9000, 300, 1000), (8200, 2050, 130), (8190, 2052, 512), (8200, 4090, 2900)])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("pad", [0, 3, 64])
def test_mx4_matmul_stores_what_is_there(m, n, k, kind, pad):
    """Many rows of short and long lines, out with rows that begin anywhere, on vectors and on whole lines: products in float64 of the values, nothing else touched."""
    _say("mx4 matmul stores", m, n, k, kind, pad)
    dtype = TYPES[kind]
    gen = torch.Generator(device=DEV).manual_seed(m + k)
    packed, values = [], []
    for rows in (m, n):
        x = torch.randn(rows, k, generator=gen, device=DEV)
        packed.append(B.mx4_empty(rows, k, DEV))
        B.adaqp_mx4_quantize(x, k, B.MX4_NEAREST, 0, packed[-1], None)
        values.append(torch.from_numpy(D.mx4_values(packed[-1][0].cpu().numpy(), packed[-1][1].cpu().numpy(), k)).to(DEV))
    ld = n + 3 if pad == 3 else -(-n // pad) * pad if pad else n
    buf = torch.full((m * ld + 64,), SENTINEL, dtype=dtype, device=DEV)
    out = buf[:m * ld].view(m, ld)
    B.adaqp_mx4_matmul(*packed, k, out[:, :n], _bytes(B.adaqp_mx4_matmul_workspace_bytes(m, n, k)).fill_(0xFF))
    want, size = values[0] @ values[1].t(), values[0].abs() @ values[1].abs().t()
    tol = 2 * U * (k / 64 + 16) * size
    if kind == "bf16":
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert bool(((out[:, :n].double() - want).abs() <= tol).all())
    line = 128 // dtype.itemsize
    written = -(-n // line) * line if ld % line == 0 else n         # whole lines, zeros behind the last column
    assert not out[:, n:written].any() and bool((out[:, written:] == SENTINEL).all()) and bool((buf[m * ld:] == SENTINEL).all())


def test_mx4_matmul_of_extreme_scales_nan_blocks_and_nothing():
    (ac, asc), av = _mx_random(40, 200, 1)
    (bc, bsc), bv = _mx_random(50, 200, 2)
    asc[0, 3, 1], bsc[1, 7, 2] = 255, 255           # row 3 and column 7; columns 192..199 lie in block 6
    asc[1, 5, 2] = 0
    asc[0, 9], bsc[0, 9] = 250, 10                  # far from 1, together near it
    out = torch.empty(40, 50, device=DEV)
    B.adaqp_mx4_matmul((ac, asc), (bc, bsc), 200, out, _bytes(B.adaqp_mx4_matmul_workspace_bytes(40, 50, 200)))
    av, bv = D.mx4_values(ac.cpu().numpy(), asc.cpu().numpy(), 200), D.mx4_values(bc.cpu().numpy(), bsc.cpu().numpy(), 200)
    want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
    got = _np(out)
    nan = np.isnan(want)
    assert nan[3].all() and nan[:, 7].all() and np.array_equal(np.isnan(got), nan)
    fine = ~nan & (size < 3e38)                     # elsewhere a partial sum may pass fp32's range
    assert fine[9, 9] and np.all(np.abs(got - want)[fine] <= 2 * U * 24 * size[fine])
    out.fill_(SENTINEL)
    B.adaqp_mx4_matmul(B.mx4_empty(40, 0, DEV), B.mx4_empty(50, 0, DEV), 0, out, None)
    assert not out.any()
    B.adaqp_mx4_matmul(B.mx4_empty(0, 32, DEV), B.mx4_empty(50, 32, DEV), 32, torch.empty(0, 50, device=DEV), None)


def test_mx4_gradients_of_a_product_are_differences():
    """Operands that 4 bits hold exactly both ways: the three products of a layer are then exact, and the gradients are slopes of sum(dz * z)."""
    rng = np.random.default_rng(8)
    rows, k, n = 96, 70, 40
    x, w, dz = (D.VALUES[rng.integers(0, 8, size=s)] * rng.choice([-1, 1], size=s) for s in ((rows, k), (n, k), (rows, n)))
    for v in (x, w, dz):                            # a 6 in each block of either direction, or a block's scale would double what is below 4
        v[::8, :] = 6
        v[:, ::8] = 6
    packed = {}
    for name, v in (("x", x), ("w", w), ("dz", dz)):
        m = _matrix(v, torch.float32)
        packed[name], packed[name + "t"] = B.mx4_empty(*v.shape, DEV), B.mx4_empty(*v.shape[::-1], DEV)
        B.adaqp_mx4_quantize(m, v.shape[1], B.MX4_STOCHASTIC, 5, packed[name], packed[name + "t"])
    z, dx, dw = (torch.empty(s, device=DEV) for s in ((rows, n), (rows, k), (n, k)))
    for a, b, depth, out in (("x", "w", k, z), ("dz", "wt", n, dx), ("dzt", "xt", rows, dw)):
        B.adaqp_mx4_matmul(packed[a], packed[b], depth, out, _bytes(B.adaqp_mx4_matmul_workspace_bytes(out.shape[0], out.shape[1], depth)))
    assert np.array_equal(_np(z), x @ w.T)
    for _ in range(3):
        vx, vw = rng.integers(-3, 4, size=x.shape), rng.integers(-3, 4, size=w.shape)
        slope = ((dz * ((x + vx) @ w.T)).sum() - (dz * ((x - vx) @ w.T)).sum() + (dz * (x @ (w + vw).T)).sum() - (dz * (x @ (w - vw).T)).sum()) / 2
        assert (_np(dx) * vx).sum() + (_np(dw) * vw).sum() == slope


# ---- orthogonalised updates ------------------------------------------------------------------------------------------------------------------------------

UPDATES = [(1, 1, 1), (1, 1, 7), (1, 7, 1), (2, 16, 16), (3, 41, 256), (3, 256, 41), (1, 64, 64), (1, 65, 130), (2, 100, 300), (1, 256, 256), (1, 602, 256),
           (1, 256, 602), (4, 127, 129), (1, 513, 700), (1, 1100, 1030), (70, 40, 50), (40, 130, 257),
           (5, 20, 33), (2, 64, 480), (2, 64, 512), (1, 960, 30), (1, 33, 100), (1, 65, 65), (2, 1500, 1400)]


def _gradient(count, rows, cols, seed):
    rng = np.random.default_rng(seed)
    rank = min(rows, cols)
    g = (rng.standard_normal((count, rows, rank)) / np.arange(1, rank + 1)) @ rng.standard_normal((count, rank, cols))
    return (g + 0.05 * rng.standard_normal((count, rows, cols))) * 1e-3


def _off(got, want):
    return np.sqrt(((got - want) ** 2).sum())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("count,rows,cols", UPDATES)
def test_orthogonalize(count, rows, cols, kind):
    """No further from the 64-bit result than four times what the same steps in plain fp32 are, and the rounding of the output."""
    _say("orthogonalize", count, rows, cols, kind)
    dtype = TYPES[kind]
    g = torch.from_numpy(_gradient(count, rows, cols, rows + cols)).to(dtype).to(DEV)
    out = torch.empty_like(g)
    work = _bytes(B.adaqp_orthogonalize_workspace_bytes(count, rows, cols)).fill_(0xFF)
    B.adaqp_orthogonalize(g, out, STEPS, 1e-7, work)
    got, values = _np(out), _np(g)
    for i in range(count):
        want = D.orthogonalize(values[i], STEPS, 1e-7)
        size = np.sqrt((want ** 2).sum())
        plain = _off(D.orthogonalize(values[i], STEPS, 1e-7, np.float32), want)
        assert _off(got[i], want) <= 4 * plain + 4 * U * size + (2.0 ** -8 if kind == "bf16" else 0) * size, i
    again = torch.empty_like(out)
    B.adaqp_orthogonalize(g, again, STEPS, 1e-7, work)
    assert torch.equal(again, out)
    B.adaqp_orthogonalize(g, g, STEPS, 1e-7, work)   # in place
    assert torch.equal(g, out)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("ld,offset", [(300, 0), (320, 0), (257, 3)])
def test_orthogonalize_pitches(ld, offset, kind):
    _say("orthogonalize pitches", ld, offset, kind)
    dtype = TYPES[kind]
    g = _matrix(_gradient(1, 100, 257, 3)[0], dtype, ld, offset)
    dense, work = torch.empty(100, 257, dtype=dtype, device=DEV), _bytes(B.adaqp_orthogonalize_workspace_bytes(1, 100, 257))
    B.adaqp_orthogonalize(g.contiguous(), dense, STEPS, 1e-7, work)
    out, buf = _out(100, 257, dtype, ld, offset)
    B.adaqp_orthogonalize(g, out, STEPS, 1e-7, work)
    assert torch.equal(out, dense)
    _untouched(buf, out, 100, 257, ld, offset, dtype)


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1e30])
def test_orthogonalize_does_not_depend_on_the_gradients_size(scale):
    """Sums of squares beyond fp32; eps 0."""
    g = _gradient(1, 60, 90, 1)[0].astype(np.float32).astype(np.float64) * 1000
    power = 2.0 ** round(np.log2(scale))
    out = [torch.empty(60, 90, device=DEV) for _ in range(2)]
    work = _bytes(B.adaqp_orthogonalize_workspace_bytes(1, 60, 90))
    for o, s in zip(out, (1.0, power)):
        B.adaqp_orthogonalize(_matrix(g * s, torch.float32), o, STEPS, 0.0, work)
    assert torch.equal(out[0], out[1])


def test_orthogonalize_other_steps_zeros_and_what_is_not_finite():
    g = _gradient(3, 50, 80, 2)
    g[1] = 0.0
    g[2, 3, 4] = np.nan
    gd = torch.from_numpy(g).float().to(DEV)
    out, work = torch.empty_like(gd), _bytes(B.adaqp_orthogonalize_workspace_bytes(3, 50, 80))
    cubic = ((1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (-1.0, 0.0, 0.0))
    for steps in ((), cubic[:1], cubic):
        B.adaqp_orthogonalize(gd, out, steps, 1e-7, work)
        got, want = _np(out), D.orthogonalize(_np(gd[0]), steps, 1e-7)
        plain = _off(D.orthogonalize(_np(gd[0]), steps, 1e-7, np.float32), want)
        assert _off(got[0], want) <= 4 * plain + 4 * U * np.sqrt((want ** 2).sum())
        assert not got[1].any() and np.isnan(got[2]).all()


# ---- streams ---------------------------------------------------------------------------------------------------------------------------------------------

def test_calls_follow_their_stream():
    """On a stream of their own, behind work that makes their inputs there."""
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(3)
    x = _matrix(rng.standard_normal((5000, 300)), torch.float32)
    want = torch.empty_like(x)
    B.adaqp_layernorm_forward(x * 3, 300, None, None, 1e-5, want)
    g = _matrix(rng.standard_normal((100, 200)), torch.float32)
    turned, work = torch.empty_like(g), _bytes(B.adaqp_orthogonalize_workspace_bytes(1, 100, 200))
    B.adaqp_orthogonalize(g * 3, turned, STEPS, 1e-7, work)
    packed, values = B.mx4_empty(5000, 300, DEV), torch.empty_like(x)
    B.adaqp_mx4_quantize(x * 3, 300, B.MX4_NEAREST, 0, packed, None)
    B.adaqp_mx4_dequantize(packed, 300, values)
    product, need = torch.empty(100, 5000, device=DEV), _bytes(B.adaqp_mx4_matmul_workspace_bytes(100, 5000, 300))
    some = (packed[0][:100].contiguous(), packed[1][:, :100].contiguous())
    B.adaqp_mx4_matmul(some, packed, 300, product, need)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            busy = torch.randn(2000, 2000, device=DEV) @ torch.randn(2000, 2000, device=DEV)
        tripled, tripled_g = x * 3, g * 3
        y, o, p, v, q = torch.empty_like(x), torch.empty_like(g), B.mx4_empty(5000, 300, DEV), torch.empty_like(x), torch.empty_like(product)
        B.adaqp_layernorm_forward(tripled, 300, None, None, 1e-5, y)
        B.adaqp_orthogonalize(tripled_g, o, STEPS, 1e-7, work)
        B.adaqp_mx4_quantize(tripled, 300, B.MX4_NEAREST, 0, p, None)
        B.adaqp_mx4_dequantize(p, 300, v)
        B.adaqp_mx4_matmul((p[0][:100].contiguous(), p[1][:, :100].contiguous()), p, 300, q, need)
        ok = torch.stack([(y == want).all(), (o == turned).all(), (v == values).all(), (q == product).all()])
    stream.synchronize()
    assert ok.cpu().tolist() == [True] * 4 and busy is not None


def test_calls_can_be_captured():
    """One graph of all calls, replayed on inputs that change, between the program's own work: every replay as the calls themselves."""
    rows, n_in, n_out = 700, 300, 64
    x, dy = torch.zeros(rows, n_in, device=DEV), torch.zeros(rows, n_out, device=DEV)
    w4, w4t = B.mx4_empty(n_out, n_in, DEV), B.mx4_empty(n_in, n_out, DEV)
    B.adaqp_mx4_quantize(torch.randn(n_out, n_in, device=DEV), n_in, B.MX4_NEAREST, 0, w4, w4t)
    x4, xt4, dz4, dzt4 = (B.mx4_empty(*s, DEV) for s in ((rows, n_in), (n_in, rows), (rows, n_out), (n_out, rows)))
    z, y, dz, dx = (torch.zeros(rows, c, device=DEV) for c in (n_out, n_out, n_out, n_in))
    stats, dgamma, dbeta, dw, turned = (torch.zeros(*s, device=DEV) for s in ((rows, 2), (n_out,), (n_out,), (n_out, n_in), (n_out, n_in)))
    work = _bytes(max(B.adaqp_mx4_matmul_workspace_bytes(rows, n_out, n_in), B.adaqp_mx4_matmul_workspace_bytes(n_out, n_in, rows),
                      B.adaqp_mx4_matmul_workspace_bytes(rows, n_in, n_out), B.adaqp_layernorm_workspace_bytes(rows, n_out),
                      B.adaqp_orthogonalize_workspace_bytes(1, n_out, n_in)))

    def calls():
        B.adaqp_mx4_quantize(x, n_in, B.MX4_NEAREST, 0, x4, xt4)
        B.adaqp_mx4_matmul(x4, w4, n_in, z, work)
        B.adaqp_layernorm_forward(z, n_out, None, None, 1e-5, y, stats)
        B.adaqp_layernorm_backward(z, dy, n_out, stats, None, dz, dgamma, dbeta, work)
        B.adaqp_mx4_quantize(dz, n_out, B.MX4_STOCHASTIC, 7, dz4, dzt4)
        B.adaqp_mx4_matmul(dz4, w4t, n_out, dx, work)
        B.adaqp_mx4_matmul(dzt4, xt4, rows, dw, work)
        B.adaqp_orthogonalize(dw, turned, STEPS, 1e-7, work)

    x.normal_()
    dy.normal_()
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for replay in range(4):
        x.normal_()
        dy.normal_()
        graph.replay()
        got = [t.clone() for t in (y, dgamma, dbeta, dx, dw, turned)]
        torch.cuda.synchronize()
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dgamma, dbeta, dx, dw, turned))), replay
        assert float(turned.abs().sum()) > 0
