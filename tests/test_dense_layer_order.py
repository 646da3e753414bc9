"""In which order DenseLayer's calls may come, on the CPU: the library's calls are replaced by ones that note their arguments."""
import pytest

torch = pytest.importorskip("torch")

from paper_2306_01381_amd import binding as B                      # noqa: E402
from paper_2306_01381_amd.dense import DenseLayer                  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    noted = []
    for name in ("adaqp_mx4_quantize", "adaqp_mx4_matmul", "adaqp_layernorm_forward", "adaqp_layernorm_backward", "adaqp_orthogonalize"):
        monkeypatch.setattr(B, name, lambda *args, name=name, **kw: noted.append((name, args)))
    return noted


def test_backward_wants_the_columns_of_its_own_forward(calls):
    """x's columns' form, which dW is a product with, is made in a forward that trains; another's is never taken for it."""
    layer = DenseLayer(20, 8, 4, "cpu")
    x, dy = torch.zeros(20, 8), torch.zeros(20, 4)

    def refused():
        before = len(calls)
        with pytest.raises(RuntimeError):
            layer.backward(dy)
        with pytest.raises(RuntimeError):
            layer.backward(dy, wants_dx=False)
        assert len(calls) == before and layer.steps == steps

    steps = 0
    refused()                                       # before any forward
    layer.forward(x, training=False)
    refused()
    layer.forward(x)                                # train, evaluate, train
    layer.backward(dy)
    steps = 1
    layer.backward(dy, wants_dx=False)              # again from the same forward
    steps = 2
    layer.update(0.1)
    layer.forward(x, training=False)
    refused()
    layer.forward(x)
    layer.backward(dy)
    assert layer.steps == 3


def test_layers_round_by_numbers_of_their_own(calls):
    """A gradient that one layer rounded is what the next rounds again: with the same numbers its error would not be independent.  The numbers of a call are those of its
    seed (rows) and the one behind it (columns)."""
    def taken(layer, steps=200):
        layer.forward(torch.zeros(20, 8))
        calls.clear()
        for _ in range(steps):
            layer.backward(torch.zeros(20, 8))
        seeds = [args[3] % 2 ** 64 for name, args in calls if name == "adaqp_mx4_quantize"]
        assert len(seeds) == steps
        return {s for seed in seeds for s in (seed, (seed + 1) % 2 ** 64)}

    sets = [taken(DenseLayer(20, 8, 8, "cpu")) for _ in range(4)] + [taken(DenseLayer(20, 8, 8, "cpu", seed=s)) for s in (1 << 40, (1 << 40) + 1, (1 << 40) + 3, 2 ** 63 - 1)]
    assert all(len(s) == 400 for s in sets)
    for i, a in enumerate(sets):
        for b in sets[:i]:
            assert not a & b
    assert taken(DenseLayer(20, 8, 8, "cpu", seed=5)) == taken(DenseLayer(20, 8, 8, "cpu", seed=5))     # and can be had again


def test_layers_begin_with_weights_of_their_own(calls):
    a, b = DenseLayer(20, 8, 8, "cpu"), DenseLayer(20, 8, 8, "cpu")
    assert not torch.equal(a.weight, b.weight)
    assert torch.equal(DenseLayer(20, 8, 8, "cpu", seed=5).weight, DenseLayer(20, 8, 8, "cpu", seed=5).weight)
