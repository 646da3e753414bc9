"""In which order the calls of DenseLayer's 8-bit form, Embedding and ClassLoss may come, on the CPU: the library's calls are replaced by ones that note their arguments."""
import pytest

torch = pytest.importorskip("torch")

from paper_2306_01381_amd import binding as B                      # noqa: E402
from paper_2306_01381_amd.dense import ClassLoss, DenseLayer, Embedding  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    noted = []
    for name in B.EXPORTS:
        if name.startswith(("adaqp_mx4_", "adaqp_f8_", "adaqp_layernorm_", "adaqp_orthogonalize", "adaqp_embedding_", "adaqp_dropout", "adaqp_logprob_")) and not name.endswith("_bytes"):
            monkeypatch.setattr(B, name, lambda *args, name=name, **kw: noted.append((name, args)))
    return noted


def test_a_layer_has_operands_of_4_or_8_bits_and_drops_less_than_all():
    for wrong in (dict(bits=16), dict(bits=0), dict(drop=-0.1), dict(drop=1.0), dict(drop=float("nan"))):
        with pytest.raises(ValueError):
            DenseLayer(20, 8, 4, "cpu", **wrong)


def test_products_are_of_the_layers_bits(calls):
    for bits, family in ((4, "adaqp_mx4_"), (8, "adaqp_f8_")):
        calls.clear()
        layer = DenseLayer(20, 8, 4, "cpu", bits=bits)
        layer.forward(torch.zeros(20, 8))
        layer.backward(torch.zeros(20, 4))
        layer.update(0.1)
        names = {name for name, _ in calls if name.startswith(("adaqp_mx4_", "adaqp_f8_"))}
        assert names == {family + "quantize", family + "matmul"}


def test_dropped_elements_are_those_of_the_last_forward(calls):
    """Backward drops what the last training forward dropped; evaluating drops nothing and takes no numbers; layers and forwards have numbers of their own."""
    def seeds():
        found = [args[3] % 2 ** 64 for name, args in calls if name == "adaqp_dropout"]
        calls.clear()
        return found
    x, dy = torch.zeros(20, 8), torch.zeros(20, 8)
    layer, other = DenseLayer(20, 8, 8, "cpu", drop=0.5), DenseLayer(20, 8, 8, "cpu", drop=0.5)
    seeds()
    layer.forward(x)
    layer.backward(dy)
    layer.backward(dy, wants_dx=False)
    first = seeds()
    assert len(first) == 3 and len(set(first)) == 1
    layer.forward(x, training=False)
    assert seeds() == []
    with pytest.raises(RuntimeError):
        layer.backward(dy)
    layer.forward(x)
    layer.backward(dy)
    second = seeds()
    other.forward(x)
    assert len(set(second)) == 1 and len({first[0], second[0], seeds()[0]}) == 3
    plain = DenseLayer(20, 8, 8, "cpu")
    plain.forward(x)
    plain.backward(dy)
    assert seeds() == []


def test_gradients_of_an_embedding_want_sorted_ids(calls):
    nodes, ids, dy = Embedding(10, 6, 5, "cpu"), torch.zeros(5, dtype=torch.int32), torch.zeros(5, 6)

    def refused():
        before = len(calls)
        for call in (lambda: nodes.backward(dy), lambda: nodes.descend(dy, 0.1)):
            with pytest.raises(RuntimeError):
                call()
        assert len(calls) == before
    refused()
    nodes.forward(ids, training=False)
    refused()
    nodes.forward(ids)
    nodes.backward(dy)
    nodes.descend(dy, 0.1)
    assert [name for name, _ in calls] == ["adaqp_embedding_forward"] * 2 + ["adaqp_embedding_sort"] + ["adaqp_embedding_backward"] * 2
    nodes.forward(ids, training=False)
    refused()
    with pytest.raises(ValueError):
        Embedding(10, 6, 5, "cpu", table=torch.zeros(9, 6))


def test_the_loss_divides_by_the_rows_that_have_a_class(calls):
    loss = ClassLoss(20, 4, "cpu")
    loss.forward(torch.zeros(20, 4), torch.zeros(20, dtype=torch.int32))
    loss.backward(torch.zeros(20, 4), torch.zeros(20, dtype=torch.int32), 8)
    assert calls[-1][0] == "adaqp_logprob_backward" and calls[-1][1][7] == -1.0 / 8


def test_backward_drops_what_forward_dropped_though_the_share_has_changed_since(calls):
    x, dy = torch.zeros(20, 8), torch.zeros(20, 8)

    def shares():
        found = [args[2] for name, args in calls if name == "adaqp_dropout"]
        calls.clear()
        return found
    layer = DenseLayer(20, 8, 8, "cpu", drop=0.5)
    layer.forward(x)
    layer.drop = 0.25
    layer.backward(dy)
    assert shares() == [0.5, 0.5]
    layer.forward(x)
    layer.drop = 0.0
    layer.backward(dy)
    assert shares() == [0.25, 0.25]
    layer.forward(x)
    layer.drop = 0.5
    layer.backward(dy)
    assert shares() == []


def test_the_loss_of_a_batch_without_given_classes_has_no_slope(calls):
    loss, logits, none = ClassLoss(20, 4, "cpu"), torch.zeros(20, 4), torch.full((20,), -1, dtype=torch.int32)
    loss.forward(logits, none)
    assert loss.backward(logits, none, 0) is loss.dlogits
    assert calls[-1][0] == "adaqp_logprob_backward" and calls[-1][1][7] == 0.0
    before = len(calls)
    with pytest.raises(ValueError):
        loss.backward(logits, none, -1)
    assert len(calls) == before
