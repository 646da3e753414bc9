"""The dense operators at sizes whose launches pass 2^32 threads or whose places pass 32 bits.  Parts of the results are compared with calls of few rows, which the other
tests compare with the definitions.  Each test says how much device memory it needs and is skipped where there is less."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
GIB = 1 << 30
U = 2.0 ** -24


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


def _need(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < (gib + 4) * GIB:
        pytest.skip(f"{free // GIB} GiB of device memory are free, {gib + 4} are needed")


def _parts(n, step=1 << 24):
    """The first and the last rows, those around 2^31 bytes, 2^32 threads and the like, and some between."""
    return [(at, min(at + step, n)) for at in range(0, n, step)]


def _random(shape, low, high, gen):
    """Random bytes, filled in pieces of at most 2^30."""
    t = torch.empty(shape, dtype=torch.uint8, device=DEV)
    flat = t.view(-1)
    for at in range(0, flat.numel(), 1 << 30):
        flat[at:at + (1 << 30)].random_(low, high, generator=gen)
    return t


def test_dequantize_of_more_than_2_32_granules():
    rows, cols = (1 << 28) + 3, 128
    _need(83)
    _say("dequantize large", rows, cols)
    gen = torch.Generator(device=DEV).manual_seed(1)
    codes, scales = _random((rows, 64), 0, 256, gen), _random((1, rows, 4), 100, 150, gen)
    out = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device=DEV)
    B.adaqp_mx4_dequantize((codes, scales), cols, out)
    for a, b in _parts(rows):
        some = torch.empty(b - a, cols, dtype=torch.bfloat16, device=DEV)
        B.adaqp_mx4_dequantize((codes[a:b], scales[:, a:b]), cols, some)
        assert torch.equal(out[a:b], some), a


def test_product_of_few_rows_with_more_than_2_28():
    m, n, k = 3, (1 << 28) + 5, 96
    _need(21)
    _say("product large, few rows", m, n, k)
    gen = torch.Generator(device=DEV).manual_seed(2)
    a = B.mx4_empty(m, k, DEV)
    B.adaqp_mx4_quantize(torch.randn(m, k, generator=gen, device=DEV), k, B.MX4_NEAREST, 0, a, None)
    codes, scales = _random((n, 64), 0, 256, gen), _random((1, n, 4), 120, 130, gen)
    for at in range(0, n, 1 << 24):
        codes[at:at + (1 << 24), k // 2:] = 0       # behind the last column
    assert B.adaqp_mx4_matmul_workspace_bytes(m, n, k) == 0
    out = torch.full((m, n), float("nan"), device=DEV)
    B.adaqp_mx4_matmul(a, (codes, scales), k, out, None)
    for first, last in _parts(n):
        some = torch.empty(m, last - first, device=DEV)
        B.adaqp_mx4_matmul(a, (codes[first:last], scales[:, first:last]), k, some, None)
        assert torch.equal(out[:, first:last], some), first


def test_as_many_rows_as_there_may_be():
    """2^31 - 1 rows of one column: quantised, and multiplied with one row."""
    rows = (1 << 31) - 1
    _need(158)
    _say("most rows", rows)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device=DEV)
    for a, b in _parts(rows, 1 << 28):
        x[a:b].normal_(generator=gen)
    packed = B.mx4_empty(rows, 1, DEV)
    B.adaqp_mx4_quantize(x, 1, B.MX4_NEAREST, 0, packed, None)
    one = B.mx4_empty(1, 1, DEV)
    B.adaqp_mx4_quantize(torch.full((1, 1), 3.0, device=DEV), 1, B.MX4_NEAREST, 0, one, None)
    out = torch.full((rows, 1), float("nan"), device=DEV)
    B.adaqp_mx4_matmul(packed, one, 1, out, None)
    for a, b in _parts(rows, 1 << 26):
        some, values = B.mx4_empty(b - a, 1, DEV), torch.empty(b - a, 1, device=DEV)
        B.adaqp_mx4_quantize(x[a:b], 1, B.MX4_NEAREST, 0, some, None)
        assert torch.equal(packed[0][a:b], some[0]) and torch.equal(packed[1][:, a:b], some[1]), a
        B.adaqp_mx4_dequantize(some, 1, values)
        assert torch.equal(out[a:b], values.mul_(3.0)), a


@pytest.mark.parametrize("rows,dim", [(3, (1 << 26) + 37), (2, 1 << 26)])
def test_layernorm_gradients_of_more_than_2_26_columns(rows, dim):
    _need(8)
    _say("layernorm large", rows, dim)
    gen = torch.Generator(device=DEV).manual_seed(4)
    x, dy = (torch.randn(rows, dim, generator=gen, device=DEV) for _ in range(2))
    gamma = 1 + 0.1 * torch.randn(dim, generator=gen, device=DEV)
    mean = x.double().mean(1)
    stats = torch.stack([mean, (x.double().var(1, unbiased=False) + 1e-5).rsqrt()], 1).float()
    dx, dgamma, dbeta = torch.full_like(x, float("nan")), torch.full((dim,), float("nan"), device=DEV), torch.full((dim,), float("nan"), device=DEV)
    work = torch.empty(B.adaqp_layernorm_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV)
    B.adaqp_layernorm_backward(x, dy, dim, stats, gamma, dx, dgamma, dbeta, work)
    mean, rstd = stats.double().unbind(1)
    k = dim / 256 + 56                              # terms that a lane adds one after the other, and the joins
    want_gamma, want_beta, of_gamma, of_beta = (torch.zeros(dim, dtype=torch.float64, device=DEV) for _ in range(4))
    for r in range(rows):
        h = (x[r].double() - mean[r]) * rstd[r]
        d = dy[r].double()
        g = d * gamma.double()
        want = rstd[r] * (g - g.mean() - h * (g * h).mean())
        tol = rstd[r] * U * (8 * g.abs() + k * g.abs().mean() + (k + 8) * h.abs() * (g * h).abs().mean())
        assert bool(((dx[r].double() - want).abs() <= tol + U * (want.abs() + tol)).all()), r
        want_gamma += d * h
        want_beta += d
        of_gamma += (d * h).abs()
        of_beta += d.abs()
    assert bool(((dgamma.double() - want_gamma).abs() <= (rows + 4) * U * of_gamma).all())
    assert bool(((dbeta.double() - want_beta).abs() <= rows * U * of_beta).all())
