"""The dense operators at the ends of their ranges: what is not finite, the largest magnitudes."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dense as D                                        # noqa: E402
from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
STEPS = ((3.4445, -4.7750, 2.0315),) * 5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def _say(*what):
    print(*what, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("rows,cols", [(50, 80), (33, 7), (200, 130), (700, 650)])
def test_orthogonalize_of_what_is_not_finite(rows, cols, steps, bad, kind):
    """One bad element makes its matrix NaN throughout, with and without steps, in every form; its neighbours keep their values."""
    _say("orthogonalize not finite", rows, cols, steps, bad, kind)
    gen = torch.Generator(device=DEV).manual_seed(rows)
    g = torch.randn(3, rows, cols, generator=gen, device=DEV).to(kind)
    work = torch.empty(max(1, B.adaqp_orthogonalize_workspace_bytes(3, rows, cols)), dtype=torch.uint8, device=DEV)
    want, got = torch.empty_like(g), torch.empty_like(g)
    B.adaqp_orthogonalize(g, want, STEPS[:steps], 1e-7, work)
    g[1, rows // 2, cols - 1] = bad
    B.adaqp_orthogonalize(g, got, STEPS[:steps], 1e-7, work)
    assert bool(got[1].isnan().all())
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and bool(want.isfinite().all())


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(40, 200), (64, 64), (33, 31)])
def test_stochastic_codes_of_the_largest_magnitudes_are_finite(rows, cols, kind):
    """Beyond 1.5 * 2^127 the next of the codes' values may be 2^128, which fp32 does not have: 3 * 2^126 is taken.  Everything else as defined, by rows and by columns."""
    _say("mx4 largest", rows, cols, kind)
    rng = np.random.default_rng(cols)
    x = rng.uniform(-1, 1, size=(rows, cols)) * rng.choice([2.0 ** 127.99, 2.0 ** 127, 2.0 ** 126, 2.0 ** 124], size=(rows, cols))
    largest = float(torch.finfo(kind).max)
    x[::3, ::5], x[1::7, 1::4] = largest, -largest
    xd = torch.from_numpy(x).to(kind).clamp_(-largest, largest).to(DEV)
    x = xd.double().cpu().numpy()
    assert np.isfinite(x).all()
    for seed in (1, 77, 2 ** 40 + 3):
        packed, packed_t = B.mx4_empty(rows, cols, DEV), B.mx4_empty(cols, rows, DEV)
        B.adaqp_mx4_quantize(xd, cols, B.MX4_STOCHASTIC, seed, packed, packed_t)
        alone = B.mx4_empty(rows, cols, DEV)
        B.adaqp_mx4_quantize(xd, cols, B.MX4_STOCHASTIC, seed, alone, None)
        for got, want in ((packed, D.mx4_quantize(x, seed)), (packed_t, D.mx4_quantize(x.T, seed + 1)), (alone, D.mx4_quantize(x, seed))):
            assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
        back = torch.empty(rows, cols, dtype=kind, device=DEV)
        B.adaqp_mx4_dequantize(packed, cols, back)
        assert bool(back.isfinite().all()) and float(back.abs().max()) == 1.5 * 2.0 ** 127


def test_evaluating_between_steps_changes_nothing():
    """Train, evaluate other rows, train: the same bits as without the evaluation."""
    from paper_2306_01381_amd.dense import DenseLayer
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, other, dy = (torch.randn(300, c, generator=gen, device=DEV) for c in (70, 70, 41))
    layers = [DenseLayer(300, 70, 41, DEV, seed=9) for _ in range(2)]
    for step in range(2):
        for layer, evaluates in zip(layers, (False, True)):
            if evaluates:
                layer.forward(other, training=False)
            layer.forward(x)
            layer.backward(dy)
            layer.update(0.02, 0.9, 0.1)
        for name in ("y", "dx", "dweight", "dgamma", "dbeta", "weight", "gamma", "beta"):
            assert torch.equal(*(getattr(layer, name) for layer in layers)), (step, name)
    assert float(layers[0].dweight.abs().max()) > 0
