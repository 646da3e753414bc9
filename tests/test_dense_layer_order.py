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
