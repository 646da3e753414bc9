"""Log probabilities of rows whose masks are finite: every logit of a lane, of a split or of a row but one may be the type's lowest value, or one that is merely far below the others."""
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
LOWEST = "lowest"                                    # of the type
# Rows are held in registers up to 2048 classes, walked by four waves beyond, and split from 8192 on where there are fewer than 512 of them.
CLASSES = [41, 2048, 2049, 3000, 8191, 8192, 20_000, 65_537]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.empty_cache()


def _np(t):
    return t.double().cpu().numpy()


def _vec(v, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(v)).to(dtype).to(DEV)


def _rows(classes, mask, rng):
    x = 3 * rng.standard_normal((12, classes))
    x[0, :classes // 2] = mask                       # before the others
    x[1, classes // 2:] = mask                       # behind them
    x[2, np.arange(classes) % 1000 != 7] = mask      # a few are allowed
    x[3, :-1] = mask                                 # the last is
    x[4, 1:] = mask                                  # the first is
    x[5] = mask                                      # none is, and all are equal
    x[6, rng.random(classes) < 0.99] = mask
    x[7, :classes // 2], x[7, classes // 2:] = mask, mask / 2
    x[8, classes // 3] = -mask                       # one far above the others
    x[9, [1, classes // 3, classes - 1]] = -mask     # three, equal
    x[10] = mask * (1 - rng.integers(0, 3, classes) / 4)
    x[11, ::2], x[11, 1::2] = mask, -np.inf          # ruled out both ways
    return x


def _tolerances(x, rest):
    """Of rest and entropy.  exp of u = x - max is off by (2 |u| + 4) u, relatively (u's own rounding, the product with log2 e, the instruction); at each of at most classes / 512 + 24 joins a part is
    multiplied by such an exp, of differences whose sum is at most the range of what counts, below 104; additions: classes / 64 + 40 in turn."""
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


def _close(got, want, tol):
    """Within tol, or what fp32 makes of a number beyond its range."""
    with np.errstate(invalid="ignore", over="ignore"):
        return (np.abs(got - want) <= tol) | (got == want.astype(np.float32))


@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e12, -1e20, -1e30, -2e38, -3e38, LOWEST, 1e12, 3e38])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("classes", CLASSES)
def test_logprob_of_finite_masks(classes, kind, mask):
    print("logprob masks", classes, kind, mask, flush=True)
    sys.stdout.flush()
    dtype, rng = TYPES[kind], np.random.default_rng(classes)
    x64 = _rows(classes, torch.finfo(dtype).min if mask == LOWEST else mask, rng)
    rows, n_top = x64.shape[0], 5
    xd = torch.from_numpy(x64).to(dtype).to(DEV)
    x = _np(xd)
    targets = rng.integers(0, classes, rows)
    targets[[0, 3, 4, 8, 9]] = 0, classes - 1, 1, classes // 3, 1
    td = _vec(targets, torch.int32)
    logp, entropy, stats, top_logp = (torch.full(s, SENTINEL, device=DEV) for s in ((rows,), (rows,), (rows, 2), (rows, n_top)))
    top_class = torch.empty(rows, n_top, dtype=torch.int32, device=DEV)
    work = torch.full((max(B.adaqp_logprob_workspace_bytes(rows, classes, n_top), 1),), 0xFF, dtype=torch.uint8, device=DEV)
    B.adaqp_logprob_forward(xd, classes, td, logp, entropy, stats, top_logp, top_class, work)
    want, top, rest, want_entropy = O.log_probabilities(x)
    off_rest, off_entropy = _tolerances(x, rest)
    at = np.arange(rows)
    assert np.array_equal(_np(stats)[:, 0], top)
    assert np.all(np.abs(_np(stats)[:, 1] - rest) <= off_rest)
    assert np.all(np.abs(_np(entropy) - want_entropy) <= off_entropy)
    u = np.abs(x[at, targets] - top)
    assert np.all(_close(_np(logp), want[at, targets], off_rest + U * (u + np.abs(want[at, targets]))))
    order = O.largest(x, n_top)
    assert np.array_equal(top_class.cpu().numpy(), order)
    u, tops = np.abs(np.take_along_axis(x, order, 1) - top[:, None]), np.take_along_axis(want, order, 1)
    with np.errstate(invalid="ignore"):
        assert np.all(_close(_np(top_logp), tops, off_rest[:, None] + U * (u + np.abs(tops))))
    # without the likeliest: the same bits
    only, only_stats = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    B.adaqp_logprob_forward(xd, classes, None, None, only, only_stats, workspace=work)
    assert torch.equal(only, entropy) and torch.equal(only_stats, stats)
    dlogp, dentropy = _vec(rng.standard_normal(rows)), _vec(rng.standard_normal(rows))
    given_stats, given_entropy = _np(stats), _np(entropy)
    for gl, gh in ((None, None), (dlogp, dentropy)):
        d = torch.full((rows, classes), SENTINEL, dtype=dtype, device=DEV)
        B.adaqp_logprob_backward(xd, classes, td, stats, entropy, gl, gh, 0.7, d)
        l64, h64 = np.ones(rows) if gl is None else _np(gl), np.zeros(rows) if gh is None else _np(gh)
        scale = float(np.float32(0.7))
        with np.errstate(invalid="ignore"):
            slope = O.logprob_gradient(x, targets, given_stats[:, 0], given_stats[:, 1], given_entropy, l64, h64, scale)
            far = np.abs(x - given_stats[:, :1])
            lp, p = np.minimum(far + given_stats[:, 1:], 300.0), np.exp(-(far + given_stats[:, 1:]))
        # exp(logp) is off by |u| + 3 |logp| + 4 roundings; of what it is multiplied with each rounds once.  A p below 2^-126 may be taken for zero
        rel = U * (np.minimum(far, 300.0) + 3 * lp + 8)
        H = np.abs(given_entropy)[:, None]
        one = np.zeros(p.shape)
        one[at, targets] = 1.0
        tol = scale * (np.abs(l64)[:, None] * (p * rel + 4 * U * one) + np.abs(h64)[:, None] * p * ((lp + H) * (rel + 4 * U) + U * (np.minimum(far, 300.0) + 2 * lp + H))) + 4 * U * np.abs(slope)
        tol = tol + 2.0 ** -126 * (1 + scale * (np.abs(l64)[:, None] + np.abs(h64)[:, None] * (lp + H)))
        half = 0.0 if dtype == torch.float32 else 2.0 ** -8
        assert np.all(np.abs(_np(d) - slope) <= tol + half * (np.abs(slope) + tol))
