"""CPU-only checks of what adaqp_train.h declares: sizes, refusals before any launch, and pins of the plain definitions."""
import ctypes

import numpy as np
import pytest

from oracle import train as O
from paper_2306_01381_amd import binding as B

P = 4096                                            # stands for a device pointer: nothing here reaches a launch
NAN, INF = float("nan"), float("inf")


def _refused(name, good, changes):
    """Each change of a good argument list is refused with its status; the good list itself is never called."""
    fn = getattr(B.lib(), name)
    for change, status in changes:
        args = list(good)
        for at, value in change.items():
            args[at] = value
        assert fn(*args) == status, (name, change)


def test_f8_sizes():
    assert B.adaqp_f8_code_bytes(10, 1) == 1280 and B.adaqp_f8_scale_bytes(10, 1) == 16
    assert B.adaqp_f8_code_bytes(17, 602) == 17 * 5 * 128 and B.adaqp_f8_scale_bytes(17, 602) == 5 * 32
    assert B.adaqp_f8_code_bytes(0, 5) == 0 and B.adaqp_f8_scale_bytes(7, 0) == 0
    assert B.adaqp_f8_code_bytes(-1, 5) == B.adaqp_f8_scale_bytes(5, -1) == B.adaqp_f8_code_bytes(1 << 31, 1) == -1
    for rows, cols in ((17, 602), (16, 128), (0, 5), (5, 0)):
        codes, scales = B.f8_empty(rows, cols, "cpu")
        assert codes.numel() == B.adaqp_f8_code_bytes(rows, cols) and scales.numel() == B.adaqp_f8_scale_bytes(rows, cols)


def test_workspaces():
    L, n = B.lib(), ctypes.c_int64()
    assert B.adaqp_embedding_sort_workspace_bytes(0, 8) == 0
    for ids, entries in ((1, 0), (1, 1), (5000, 600), (1 << 20, 1 << 30), ((1 << 31) - 1, (1 << 31) - 1)):
        need = B.adaqp_embedding_sort_workspace_bytes(ids, entries)
        assert need > 0 and need % 256 == 0
    assert B.adaqp_embedding_backward_workspace_bytes(0, 8) == B.adaqp_embedding_backward_workspace_bytes(8, 8) == 0
    assert B.adaqp_embedding_backward_workspace_bytes(33, 8) % 256 == 0 and B.adaqp_embedding_backward_workspace_bytes(33, 8) >= 2 * 2 * 8 * 4
    assert B.adaqp_logprob_workspace_bytes(0, 8, 0) == B.adaqp_logprob_workspace_bytes(100_000, 41, 5) == 0
    assert B.adaqp_logprob_workspace_bytes(1, 128_000, 20) > 0 and B.adaqp_logprob_workspace_bytes(1, 128_000, 20) % 256 == 0
    assert B.adaqp_f8_matmul_workspace_bytes(0, 5, 5) == 0 and B.adaqp_f8_matmul_workspace_bytes(5, 5, 0) == 0
    assert B.adaqp_f8_matmul_workspace_bytes(256, 300, 196_000) > 0
    at = ctypes.byref(n)
    assert L.adaqp_embedding_sort_workspace_bytes(-1, 8, at) == L.adaqp_embedding_sort_workspace_bytes(1, -1, at) == L.adaqp_embedding_sort_workspace_bytes(1, 1, None) == B.EINVAL
    assert L.adaqp_embedding_sort_workspace_bytes(1 << 31, 8, at) == L.adaqp_embedding_sort_workspace_bytes(8, 1 << 31, at) == B.ESIZE
    assert L.adaqp_embedding_backward_workspace_bytes(-1, 8, at) == L.adaqp_embedding_backward_workspace_bytes(1, 0, at) == L.adaqp_embedding_backward_workspace_bytes(1, 1, None) == B.EINVAL
    assert L.adaqp_embedding_backward_workspace_bytes(1 << 31, 8, at) == L.adaqp_embedding_backward_workspace_bytes(1, (1 << 30) + 1, at) == B.ESIZE
    assert L.adaqp_logprob_workspace_bytes(-1, 8, 0, at) == L.adaqp_logprob_workspace_bytes(1, 0, 0, at) == L.adaqp_logprob_workspace_bytes(1, 8, 9, at) == B.EINVAL
    assert L.adaqp_logprob_workspace_bytes(1, 80, 33, at) == L.adaqp_logprob_workspace_bytes(1, 8, -1, at) == L.adaqp_logprob_workspace_bytes(1, 8, 0, None) == B.EINVAL
    assert L.adaqp_logprob_workspace_bytes(1, (1 << 30) + 1, 0, at) == B.ESIZE
    assert L.adaqp_f8_matmul_workspace_bytes(1 << 31, 1, 1, at) == L.adaqp_f8_matmul_workspace_bytes(1, 1, (1 << 24) + 1, at) == B.ESIZE
    assert L.adaqp_f8_matmul_workspace_bytes(1, 1, 1, None) == L.adaqp_f8_matmul_workspace_bytes(1, -1, 1, at) == B.EINVAL


def test_embedding_refusals():
    good = [P, 8, 10, 8, 0, P, 4, 1.0, 2 * P, 8, 0, None]
    _refused("adaqp_embedding_forward", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: 0}, B.EINVAL), ({4: 2}, B.EINVAL), ({5: None}, B.EINVAL), ({5: P + 2}, B.EINVAL),
        ({6: -1}, B.EINVAL), ({7: NAN}, B.EINVAL), ({7: INF}, B.EINVAL), ({8: None}, B.EINVAL), ({8: P + 1, 10: 1}, B.EINVAL), ({9: 7}, B.EINVAL), ({10: -1}, B.EINVAL),
        ({2: 1 << 31}, B.ESIZE), ({6: 1 << 31}, B.ESIZE), ({3: (1 << 30) + 1, 1: 1 << 31, 9: 1 << 31}, B.ESIZE), ({1: 1 << 59, 2: 100}, B.ESIZE)])
    assert B.lib().adaqp_embedding_forward(None, 0, 10, 8, 0, None, 0, 1.0, None, 0, 0, None) == B.OK
    good = [P, 5000, 600, 2 * P, 3 * P, 4 * P, 1 << 30, None]
    _refused("adaqp_embedding_sort", good, [
        ({0: None}, B.EINVAL), ({1: -1}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: None}, B.EINVAL), ({4: None}, B.EINVAL), ({5: None}, B.EINVAL), ({5: P + 128}, B.EINVAL),
        ({0: P + 1}, B.EINVAL), ({3: P + 2}, B.EINVAL), ({4: P + 2}, B.EINVAL), ({3: P}, B.EINVAL), ({4: P}, B.EINVAL), ({4: 2 * P}, B.EINVAL),
        ({6: B.adaqp_embedding_sort_workspace_bytes(5000, 600) - 1}, B.ESIZE), ({1: 1 << 31}, B.ESIZE), ({2: 1 << 31}, B.ESIZE)])
    assert B.lib().adaqp_embedding_sort(None, 0, 600, None, None, None, 0, None) == B.OK
    good = [P, 8, 100, 8, 0, P, P, 50, 1.0, 0, 2 * P, 8, P, 1 << 20, None]
    need = B.adaqp_embedding_backward_workspace_bytes(100, 8)
    _refused("adaqp_embedding_backward", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: 0}, B.EINVAL), ({4: 2}, B.EINVAL), ({5: None}, B.EINVAL), ({6: None}, B.EINVAL),
        ({5: P + 1}, B.EINVAL), ({6: P + 2}, B.EINVAL), ({7: -1}, B.EINVAL), ({8: NAN}, B.EINVAL), ({8: -INF}, B.EINVAL), ({9: 2}, B.EINVAL), ({10: None}, B.EINVAL), ({10: P + 2}, B.EINVAL),
        ({11: 7}, B.EINVAL), ({12: None}, B.EINVAL), ({12: P + 128}, B.EINVAL), ({13: need - 1}, B.ESIZE), ({2: 1 << 31}, B.ESIZE), ({7: 1 << 31}, B.ESIZE),
        ({3: (1 << 30) + 1, 1: 1 << 31, 11: 1 << 31}, B.ESIZE), ({11: 1 << 59}, B.ESIZE)])
    assert B.lib().adaqp_embedding_backward(None, 8, 0, 8, 0, None, None, 50, 1.0, 1, None, 8, None, 0, None) == B.OK
    assert B.lib().adaqp_embedding_backward(None, 8, 5, 8, 0, None, None, 0, 1.0, 0, None, 8, None, 0, None) == B.OK


def test_dropout_refusals():
    good = [P, 8, 2 * P, 8, 4, 8, 0, 0.5, 1, 0, None, 3 * P, 8, None]
    _refused("adaqp_dropout", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: P + 2}, B.EINVAL), ({3: 7}, B.EINVAL), ({4: -1}, B.EINVAL), ({5: 0}, B.EINVAL), ({6: 3}, B.EINVAL),
        ({7: -0.1}, B.EINVAL), ({7: 1.1}, B.EINVAL), ({7: NAN}, B.EINVAL), ({9: -1}, B.EINVAL), ({10: P + 4}, B.EINVAL), ({11: None}, B.EINVAL), ({11: P + 1, 6: 1}, B.EINVAL),
        ({12: 7}, B.EINVAL), ({11: P, 12: 9}, B.EINVAL), ({11: 2 * P, 12: 9}, B.EINVAL), ({5: (1 << 30) + 1, 1: 1 << 31, 3: 1 << 31, 12: 1 << 31}, B.ESIZE), ({1: 1 << 59}, B.ESIZE)])
    assert B.lib().adaqp_dropout(None, 8, None, 0, 0, 8, 0, 0.5, 1, 0, None, None, 8, None) == B.OK


def test_f8_refusals():
    good = [P, 8, 4, 8, 0, 0, P, P, P, P, None]
    _refused("adaqp_f8_quantize", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: -1}, B.EINVAL), ({4: 3}, B.EINVAL), ({5: 2}, B.EINVAL),
        ({6: None}, B.EINVAL), ({7: None}, B.EINVAL), ({8: None}, B.EINVAL), ({9: None}, B.EINVAL), ({6: P + 4}, B.EINVAL), ({9: P + 8}, B.EINVAL),
        ({2: 1 << 31}, B.ESIZE), ({3: 1 << 31, 1: 1 << 31}, B.ESIZE)])
    assert B.lib().adaqp_f8_quantize(None, 0, 0, 8, 0, 0, None, None, None, None, None) == B.OK
    good = [P, P, 4, 8, P, 8, 0, None]
    _refused("adaqp_f8_dequantize", good, [({0: None}, B.EINVAL), ({1: None}, B.EINVAL), ({1: P + 4}, B.EINVAL), ({2: -1}, B.EINVAL), ({4: None}, B.EINVAL),
                                           ({5: 7}, B.EINVAL), ({6: 9}, B.EINVAL), ({2: 1 << 31}, B.ESIZE)])
    good = [P, P, 4, P, P, 8, 16, P, 8, 0, P, 1 << 20, None]
    _refused("adaqp_f8_matmul", good, [
        ({0: None}, B.EINVAL), ({1: None}, B.EINVAL), ({3: None}, B.EINVAL), ({4: P + 4}, B.EINVAL), ({2: -1}, B.EINVAL), ({5: -1}, B.EINVAL), ({6: -1}, B.EINVAL),
        ({7: None}, B.EINVAL), ({7: P + 2}, B.EINVAL), ({8: 7}, B.EINVAL), ({9: 2}, B.EINVAL), ({2: 1 << 31}, B.ESIZE), ({6: 1 << 31}, B.ESIZE)])
    need = B.adaqp_f8_matmul_workspace_bytes(4, 8, 100_000)
    assert need > 0                                 # one tile: k is split
    _refused("adaqp_f8_matmul", good, [({6: 100_000, 11: need - 1}, B.ESIZE), ({6: 100_000, 10: None}, B.EINVAL), ({6: 100_000, 10: P + 128}, B.EINVAL)])


def test_logprob_refusals():
    good = [P, 40, 4, 40, 0, P, P, P, P, 5, P, P, None, 0, None]
    _refused("adaqp_logprob_forward", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 39}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: 0}, B.EINVAL), ({4: 2}, B.EINVAL), ({5: None}, B.EINVAL), ({5: P + 2}, B.EINVAL),
        ({6: P + 1}, B.EINVAL), ({7: P + 2}, B.EINVAL), ({8: P + 2}, B.EINVAL), ({9: 41}, B.EINVAL), ({9: 33}, B.EINVAL), ({9: -1}, B.EINVAL), ({9: 0}, B.EINVAL), ({10: None}, B.EINVAL),
        ({11: None}, B.EINVAL), ({10: P + 2}, B.EINVAL), ({11: P + 3}, B.EINVAL), ({3: (1 << 30) + 1, 1: 1 << 31}, B.ESIZE), ({1: 1 << 59}, B.ESIZE)])
    need = B.adaqp_logprob_workspace_bytes(4, 128_000, 5)
    wide = {1: 128_000, 3: 128_000}
    _refused("adaqp_logprob_forward", good, [(wide, B.EINVAL), ({**wide, 12: P + 128, 13: need}, B.EINVAL), ({**wide, 12: P, 13: need - 1}, B.ESIZE)])
    assert B.lib().adaqp_logprob_forward(None, 0, 0, 40, 0, None, None, None, None, 0, None, None, None, 0, None) == B.OK
    good = [P, 40, 4, 40, 0, P, P, P, P, P, 1.0, 2 * P, 40, None]
    _refused("adaqp_logprob_backward", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 39}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: 0}, B.EINVAL), ({4: 2}, B.EINVAL), ({5: P + 2}, B.EINVAL), ({6: None}, B.EINVAL),
        ({6: P + 2}, B.EINVAL), ({7: None}, B.EINVAL), ({7: P + 1}, B.EINVAL), ({8: P + 2}, B.EINVAL), ({9: P + 2}, B.EINVAL), ({10: NAN}, B.EINVAL), ({10: INF}, B.EINVAL),
        ({11: None}, B.EINVAL), ({11: P + 2}, B.EINVAL), ({12: 39}, B.EINVAL), ({11: P, 12: 41}, B.EINVAL), ({3: (1 << 30) + 1, 1: 1 << 31, 12: 1 << 31}, B.ESIZE), ({12: 1 << 59}, B.ESIZE)])
    assert B.lib().adaqp_logprob_backward(None, 0, 0, 40, 0, None, None, None, None, None, 1.0, None, 0, None) == B.OK


def test_wrappers_refuse_tensors_that_are_not_what_they_name():
    """Found by the binding, before the library is asked."""
    import torch
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: B.adaqp_embedding_forward(x, 8, ids, 1.0, x), lambda: B.adaqp_embedding_sort(ids, 4, ids, ids, None), lambda: B.adaqp_dropout(x, 8, 0.5, 1, x),
                 lambda: B.adaqp_embedding_backward(x, 8, ids, ids, 1.0, False, x, None), lambda: B.adaqp_f8_quantize(x, 8, B.F8_ROWS, None, None),
                 lambda: B.adaqp_logprob_forward(x, 8, ids, None), lambda: B.adaqp_logprob_backward(x, 8, ids, x, None, None, None, 1.0, x)):
        with pytest.raises(TypeError):
            call()                                  # not on a device
    for t, dtype in ((torch.zeros(4, dtype=torch.int64), torch.int32), (torch.zeros(4, 2)[:, 0], torch.float32)):
        with pytest.raises(TypeError):
            B._flat(t, dtype, 4, "t")
    with pytest.raises(ValueError):
        B._flat(x, torch.float32, 33, "t")
    for wrong in (torch.zeros(4, 8, dtype=torch.float64), torch.zeros(8), torch.zeros(8, 4).t()):
        with pytest.raises(TypeError):
            B._cells(wrong, 1, "t")
    with pytest.raises(ValueError):
        B._cells(x, 9, "t")


def test_wrappers_refuse_tensors_of_another_device():
    class On:
        def __init__(self, index):
            self.index, self.device = index, f"cuda:{index}"

        def get_device(self):
            return self.index

    class Stream:
        device_index, cuda_stream = 1, 77
    assert B._place(Stream, On(1), None, On(1)) == 77
    for tensors in ((On(0),), (On(1), On(0)), (On(1), None, On(2))):
        with pytest.raises(ValueError):
            B._place(Stream, *tensors)
    for tensors in ((On(-1),), (On(1), On(-1)), (On(-1), On(1)), (On(-1), On(-1))):
        with pytest.raises((TypeError, ValueError)):
            B._place(Stream, *tensors)


def test_wrappers_say_that_whole_lines_are_written():
    for name in ("adaqp_embedding_forward", "adaqp_embedding_backward", "adaqp_dropout", "adaqp_f8_dequantize", "adaqp_f8_matmul", "adaqp_logprob_backward"):
        assert "128-byte lines" in getattr(B, name).__doc__, name


# ---- the definitions ---------------------------------------------------------------------------------------------------------------------

def test_dropout_numbers_are_those_of_the_codecs_generator(oracle):
    seed, first = 0x0123456789ABCDEF, (1 << 33) + 5
    got = O.drop_numbers(3, 24, seed, first)
    for row in range(3):
        for piece in range(3):
            number = first + row
            words = oracle.philox4x32_10([piece, number & 0xFFFFFFFF, number >> 32, O.DROP_TAG], [seed & 0xFFFFFFFF, seed >> 32])
            want = [int(w) >> s & 0xFFFF for w in words for s in (0, 16)]
            assert got[row, 8 * piece:8 * piece + 8].tolist() == want


def test_dropout_definition_keeps_the_mean():
    """Of n independent elements a share of t / 2^16 +- 5 sigma is dropped, and the mean of what is left times the factor is 1 to 5 sigma."""
    for p in (0.1, 0.5, 0.9):
        keep, factor = O.dropped(500, 400, p, 11)
        n, t = keep.size, round(p * 65536) / 65536
        assert abs((~keep).mean() - t) <= 5 * np.sqrt(t * (1 - t) / n)
        assert abs((keep * factor).mean() - 1) <= 5 * np.sqrt(t / (1 - t) / n)
    assert O.dropped(2, 8, 0.0, 1)[0].all() and O.dropped(2, 8, 0.0, 1)[1] == 1.0
    assert not O.dropped(2, 8, 1.0, 1)[0].any() and O.dropped(2, 8, 1.0, 1)[1] == 0.0


def test_embedding_definition_has_the_gradients_of_differences():
    """The lookup is linear: slopes of sum(dy * out) are exact but for rounding."""
    rng = np.random.default_rng(3)
    table, ids = rng.standard_normal((7, 5)), np.array([3, -1, 3, 0, 7, 6, 3])
    dy, v = rng.standard_normal((7, 5)), rng.standard_normal((7, 5))
    slope = (dy * (O.embedding(table + v, ids, 2.5) - O.embedding(table, ids, 2.5))).sum()
    assert abs((O.embedding_gradient(dy, ids, 7, 2.5) * v).sum() - slope) <= 1e-12 * (1 + abs(slope))
    assert not O.embedding_gradient(dy, ids, 7, 2.5)[[1, 2, 4, 5]].any()


def test_f8_values_are_the_formats():
    import torch
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), O.F8_VALUES, equal_nan=True)


def test_f8_definition_pins():
    """By hand: values at scale 1, ties to the even code, the smallest scale, 256 where it would be 2^128; against torch's own rounding on random values."""
    import torch
    x = np.zeros((2, 128))
    x[0, :8] = [448, 1.0625, 1.1875, -2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, -0.0, 432]      # ties go to 1, 1.25, -0, 2^-8 and (432, between 0x7D and 0x7E) 448
    codes, scales = O.f8_quantize(x)
    assert scales[0, :2].tolist() == [127, 0] and not scales[0, 2:].any()
    assert O.f8_values(codes, scales, 8)[0].tolist() == [448, 1.0, 1.25, 0.0, 2.0 ** -8, 2.0 ** -9, 0.0, 448]
    assert codes[0, 3] == codes[0, 6] == 0x80
    assert O.f8_quantize(np.full((1, 1), 448.0 * 2 ** 5))[1][0, 0] == 132 and O.f8_quantize(np.full((1, 1), 449.0 * 2 ** 5))[1][0, 0] == 133
    most = 2.0 ** 128 * (1 - 2.0 ** -24)
    codes, scales = O.f8_quantize(np.array([[most, -most, 2.0 ** 127]]))
    assert scales[0, 0] == 247 and O.f8_values(codes, scales, 3)[0].tolist() == [240 * 2.0 ** 120, -240 * 2.0 ** 120, 2.0 ** 127]
    assert O.f8_quantize(np.array([[1.75 * 2.0 ** 127]]))[1][0, 0] == 246
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((50, 300)) * np.exp2(rng.integers(-20, 9, size=(50, 1)))).astype(np.float32)
    codes, scales = O.f8_quantize(x)
    e = np.repeat(scales[:, :50].T.astype(np.float64) - 127, 128, 1)[:, :300]
    want = torch.from_numpy(x / np.exp2(e)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes[:, :300], want) and not codes[:, 300:].any()
    block = np.abs(np.pad(x, ((0, 0), (0, 84))).reshape(50, 3, 128)).max(2)
    unit = np.exp2(scales[:, :50].T.astype(np.float64) - 127)
    assert np.all(block <= 448 * unit) and np.all(block > 224 * unit)


def test_f8_tiles_hold_the_same_values_transposed():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((130, 260))
    a, b = O.f8_values(*O.f8_quantize(x, True), 260), O.f8_values(*O.f8_quantize(x.T, True), 130)
    assert np.array_equal(a, b.T)
    assert not np.array_equal(O.f8_values(*O.f8_quantize(x), 260), O.f8_values(*O.f8_quantize(x.T), 130).T)


def test_log_probability_definition_and_its_gradients_are_differences():
    """Central differences of 1e-5 are off by 1e-10 of third derivatives (about 1 here) and by 1e-11 of the sum's size: 1e-7 leaves room for both."""
    rng = np.random.default_rng(7)
    for rows, classes in ((1, 1), (4, 2), (5, 17)):
        x, v = 3 * rng.standard_normal((rows, classes)), rng.standard_normal((rows, classes))
        if classes > 2:
            x[:, 3] = -np.inf
        targets = rng.integers(0, classes, rows)
        targets[0] = -1 if rows > 1 else 0
        targets[targets == 3] = 4
        dlogp, dentropy = rng.standard_normal(rows), rng.standard_normal(rows)
        logp, top, rest, entropy = O.log_probabilities(x)
        assert np.allclose(np.exp(logp).sum(1), 1.0, atol=1e-12) and np.all(entropy >= -1e-15)

        def loss(x):
            logp, _, _, entropy = O.log_probabilities(x)
            return 0.7 * ((np.where(targets >= 0, logp[np.arange(rows), targets], 0.0) * dlogp).sum() + (entropy * dentropy).sum())
        t = 1e-5
        slope = (loss(x + t * v) - loss(x - t * v)) / (2 * t)
        d = O.logprob_gradient(x, targets, top, rest, entropy, dlogp, dentropy, 0.7)
        assert abs((d * v).sum() - slope) <= 1e-7 * (1 + np.abs(d * v).sum())


def test_largest_definition():
    x = np.array([[1.0, 3.0, -0.0, 3.0, 0.0, -np.inf, np.nan, np.inf]])
    assert O.largest(x, 8)[0].tolist() == [6, 7, 1, 3, 0, 2, 4, 5]
