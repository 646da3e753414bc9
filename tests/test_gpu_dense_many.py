"""The dense operators where a workgroup has work more than once: layer norms of more rows than a launch has places for, updates of more tiles than there are CUs.
Definitions are computed in float64 on the device.  u = 2^-24; tolerances as in test_gpu_dense.py: a sum of t terms in turn is off by at most t u of the sum of
their magnitudes, a result of bf16 by 2^-8 of itself."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEPS = ((3.4445, -4.7750, 2.0315),) * 5


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


def _matrix(rows, dim, ld, dtype, gen, scale, shift):
    m = torch.full((rows, ld), float("nan"), dtype=dtype, device=DEV)[:, :dim]
    m.copy_(torch.randn(rows, dim, generator=gen, device=DEV) * scale + shift)
    return m


# rows, columns, pitch, pitch of what is written: 8, 16, 32, 64 and 256 lanes a row, and rows walked in memory; each has three rows and more for every group of lanes in both directions
MANY = [(200_000, 16, 16, 16), (200_000, 100, 100, 100), (200_000, 31, 64, 64), (200_003, 20, 21, 21), (100_000, 200, 200, 256), (50_000, 300, 304, 304), (50_001, 301, 301, 301),
        (25_000, 602, 640, 640), (25_000, 602, 602, 602), (25_000, 1000, 1000, 1000), (25_000, 1500, 1504, 1504), (25_001, 2000, 2000, 2000), (6_200, 3000, 3000, 3000),
        (6_200, 4100, 4100, 4160), (12_300, 2051, 2051, 2051), (12_300, 2051, 2052, 2112)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,dim,ld,ld_out", MANY)
def test_layernorm_of_many_rows(rows, dim, ld, ld_out, kind):
    _say("layernorm of many rows", rows, dim, ld, ld_out, kind)
    dtype = TYPES[kind]
    off = 2.0 ** -8 if kind == "bf16" else U
    gen = torch.Generator(device=DEV).manual_seed(dim)
    scale = torch.exp2(torch.randint(-4, 5, (rows, 1), generator=gen, device=DEV).float())
    x = _matrix(rows, dim, ld, dtype, gen, scale, torch.randn(rows, 1, generator=gen, device=DEV))
    dy = _matrix(rows, dim, ld, dtype, gen, 1.0, 0.0)
    gamma, beta = 1 + 0.3 * torch.randn(dim, generator=gen, device=DEV), torch.randn(dim, generator=gen, device=DEV)
    y, dx = (torch.full((rows, ld_out), -77.0, dtype=dtype, device=DEV) for _ in range(2))
    stats, dgamma, dbeta = torch.full((rows, 2), -77.0, device=DEV), torch.full((dim,), -77.0, device=DEV), torch.full((dim,), -77.0, device=DEV)
    B.adaqp_layernorm_forward(x, dim, gamma, beta, 1e-5, y[:, :dim], stats)

    x64 = x.double()
    mean = x64.mean(1, keepdim=True)
    d = x64 - mean
    rstd = (d.square().mean(1, keepdim=True) + float(torch.tensor(1e-5))).rsqrt()
    h = d * rstd
    k = dim / 64 + 48
    off_mean = k * U * x64.abs().mean(1, keepdim=True)
    rel = (k + 8) * U + 0.5 * (off_mean * rstd) ** 2
    want = h * gamma.double() + beta.double()
    tol = gamma.double().abs() * (off_mean * rstd * (1 + rel) + h.abs() * rel) + 4 * U * ((h * gamma.double()).abs() + beta.double().abs())
    assert bool(((y[:, :dim].double() - want).abs() <= tol + off * (want.abs() + tol) + 1e-38).all())
    assert bool(((stats[:, :1].double() - mean).abs() <= off_mean).all()) and bool(((stats[:, 1:].double() - rstd).abs() <= rel * rstd).all())

    B.adaqp_layernorm_backward(x, dy, dim, stats, gamma, dx[:, :dim], dgamma, dbeta, torch.empty(B.adaqp_layernorm_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV))
    mean, rstd = stats.double()[:, :1], stats.double()[:, 1:]
    h, d = (x64 - mean) * rstd, dy.double()
    g = d * gamma.double()
    want = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    k = dim / 64 + 56
    tol = rstd * U * (8 * g.abs() + k * g.abs().mean(1, keepdim=True) + (k + 8) * h.abs() * (g * h).abs().mean(1, keepdim=True))
    assert bool(((dx[:, :dim].double() - want).abs() <= tol + off * (want.abs() + tol) + 1e-38).all())
    chain = 8 + 32 + 64 + 32                        # a lane's rows, the groups of a workgroup, the workgroups' sums by slice, the slices
    assert bool(((dgamma.double() - (d * h).sum(0)).abs() <= (chain + 4) * U * (d * h).abs().sum(0)).all())
    assert bool(((dbeta.double() - d.sum(0)).abs() <= chain * U * d.abs().sum(0)).all())

    line = 128 // dtype.itemsize
    written = -(-dim // line) * line if ld_out % line == 0 else dim
    for m in (y, dx):
        assert not m[:, dim:written].any() and bool((m[:, written:] == -77.0).all())


def _steps(g, dtype):
    flip = g.shape[0] > g.shape[1]
    x = g.double()
    x = ((x.t() if flip else x) / (x.square().sum().sqrt() + 1e-7)).to(dtype).contiguous()
    for a, b, c in STEPS:
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if flip else x).double()


# By the sizes (padded to 64) tiles of 256 x 128 in the steps and, both ways round, in the last; symmetric products cut, and uncut in tiles of 128 x 128
TILES = [(1, 2100, 4000), (1, 4000, 2100), (3, 1700, 1800), (2, 1800, 1980), (1, 2900, 2950)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("count,rows,cols", TILES)
def test_orthogonalize_of_many_tiles(count, rows, cols, kind):
    """No further from the 64-bit result than four times what the same steps in plain fp32 are, and the rounding of the output."""
    _say("orthogonalize of many tiles", count, rows, cols, kind)
    dtype = TYPES[kind]
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    rank = min(rows, cols)
    g = torch.empty(count, rows, cols, dtype=dtype, device=DEV)
    for i in range(count):
        left = torch.randn(rows, rank, generator=gen, device=DEV) / torch.arange(1, rank + 1, device=DEV)
        g[i] = (left @ torch.randn(rank, cols, generator=gen, device=DEV) + 0.05 * torch.randn(rows, cols, generator=gen, device=DEV)) * 1e-3
    buf = torch.full((count, rows, cols + 3), -77.0, dtype=dtype, device=DEV)
    out = buf[:, :, :cols]
    work = torch.empty(B.adaqp_orthogonalize_workspace_bytes(count, rows, cols), dtype=torch.uint8, device=DEV).fill_(0xFF)
    B.adaqp_orthogonalize(g, out, STEPS, 1e-7, work)
    assert bool((buf[:, :, cols:] == -77.0).all())
    for i in range(count):
        want = _steps(g[i], torch.float64)
        size, plain = float(want.norm()), float((_steps(g[i], torch.float32) - want).norm())
        assert float((out[i].double() - want).norm()) <= 4 * plain + 4 * U * size + (2.0 ** -8 if kind == "bf16" else 0) * size, i
    again = torch.empty_like(g)
    B.adaqp_orthogonalize(g, again, STEPS, 1e-7, work)
    assert torch.equal(again, out)


def test_the_stream_that_calls_take_is_the_current_one():
    """The binding asks torch for the current stream's handle in a shorter way than by a Stream object: it is the same handle, on every stream."""
    streams = [torch.cuda.default_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams + streams[::-1]:
        with torch.cuda.stream(s):
            assert (B._stream(None) or 0) == torch.cuda.current_stream().cuda_stream == s.cuda_stream
        assert (B._stream(s) or 0) == s.cuda_stream
