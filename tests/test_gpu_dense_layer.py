"""DenseLayer against its definition in float64, and the example that trains with it."""
import importlib.util
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dense as D                                        # noqa: E402
from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def _np(t):
    return t.double().cpu().numpy()


def _held(x, seed=None):
    return D.mx4_values(*D.mx4_quantize(x, seed), x.shape[1])


@pytest.mark.parametrize("rows,n_in,n_out", [(300, 70, 41), (2000, 128, 64), (517, 602, 256)])
def test_a_step_of_the_layer_is_its_definition(rows, n_in, n_out):
    """Each call's result against the definition applied to what the layer held before it, so that no rounding of a code can fall on the other side."""
    print("dense layer", rows, n_in, n_out, flush=True)
    sys.stdout.flush()
    from paper_2306_01381_amd.dense import UPDATE_STEPS, DenseLayer
    rng = np.random.default_rng(rows)
    layer = DenseLayer(rows, n_in, n_out, DEV, seed=3)
    x = torch.from_numpy(rng.standard_normal((rows, n_in))).float().to(DEV)
    dy = torch.from_numpy(rng.standard_normal((rows, n_out)) * 1e-3).float().to(DEV)
    weight = _np(layer.weight)
    y = layer.forward(x)
    x4, w4, z = _held(_np(x)), _held(weight), _np(layer.z)
    assert np.all(np.abs(z - x4 @ w4.T) <= 2 * U * (n_in / 64 + 16) * (np.abs(x4) @ np.abs(w4).T))
    want, mean, rstd = D.layernorm(z, 1.0, 0.0, np.float32(1e-5))
    assert np.max(np.abs(_np(y) - want)) <= 1e-5 * np.max(np.abs(want))
    dx = layer.backward(dy)
    dz = _np(layer.dz)
    want, dgamma, dbeta = D.layernorm_backward(z, _np(dy), *_np(layer.stats).T, 1.0)
    assert np.max(np.abs(dz - want)) <= 1e-5 * np.max(np.abs(want))
    assert np.max(np.abs(_np(layer.dgamma) - dgamma)) <= 1e-5 * np.max(np.abs(dgamma)) and np.max(np.abs(_np(layer.dbeta) - dbeta)) <= 1e-5 * np.max(np.abs(dbeta))
    seed = layer.seed + 2 * layer.steps
    by_rows, by_columns = _held(dz, seed), _held(dz.T, seed + 1)
    wt4, xt4 = _held(weight.T), _held(_np(x).T)
    assert np.all(np.abs(_np(dx) - by_rows @ wt4.T) <= 2 * U * (n_out / 64 + 16) * (np.abs(by_rows) @ np.abs(wt4).T) + 1e-38)
    assert np.all(np.abs(_np(layer.dweight) - by_columns @ xt4.T) <= 2 * U * (rows / 64 + 16) * (np.abs(by_columns) @ np.abs(xt4).T) + 1e-38)
    layer.update(0.02, 0.9, 0.1)
    direction = D.orthogonalize(_np(layer.dweight), UPDATE_STEPS, 1e-7)
    moved = weight - 0.02 * np.sqrt(max(1.0, n_out / n_in)) * direction
    assert np.sqrt(((_np(layer.weight) - moved) ** 2).sum()) <= 1e-5 * 0.02 * np.sqrt((direction ** 2).sum()) + 4 * U * np.sqrt((weight ** 2).sum())
    codes, scales = D.mx4_quantize(_np(layer.weight))
    assert np.array_equal(layer.w4[0].cpu().numpy(), codes) and np.array_equal(layer.w4[1].cpu().numpy(), scales)


def test_the_example_learns():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_layer.py")
    spec = importlib.util.spec_from_file_location("train_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    errors = example.train(steps=60, say=lambda *w: print(*w, flush=True))
    assert len(errors) == 61 and errors[-1] < 0.25 * errors[0] and np.isfinite(errors).all()
