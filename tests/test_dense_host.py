"""CPU-only checks of the dense operators: sizes, refusals before any launch, and pins of their plain definitions."""
import ctypes

import numpy as np
import pytest

from oracle import dense as D
from paper_2306_01381_amd import binding as B

STEPS = ((3.4445, -4.7750, 2.0315),) * 5
P = 4096                                            # stands for a device pointer: nothing here reaches a launch


def test_mx4_sizes():
    assert B.adaqp_mx4_code_bytes(10, 1) == 640 and B.adaqp_mx4_scale_bytes(10, 1) == 40
    assert B.adaqp_mx4_code_bytes(3, 602) == 3 * 5 * 64 and B.adaqp_mx4_scale_bytes(3, 602) == 3 * 5 * 4
    assert B.adaqp_mx4_code_bytes(0, 5) == 0 and B.adaqp_mx4_scale_bytes(7, 0) == 0
    assert B.adaqp_mx4_code_bytes(-1, 5) == B.adaqp_mx4_scale_bytes(5, -1) == B.adaqp_mx4_code_bytes(1 << 31, 1) == -1
    codes, scales = B.mx4_empty(3, 602, "cpu")
    assert codes.numel() == B.adaqp_mx4_code_bytes(3, 602) and scales.numel() == B.adaqp_mx4_scale_bytes(3, 602)


def test_workspaces():
    assert B.adaqp_layernorm_workspace_bytes(0, 8) == 0
    assert B.adaqp_layernorm_workspace_bytes(1, 8) == 256
    assert B.adaqp_orthogonalize_workspace_bytes(0, 8, 8) == 0
    for sizes in ((1, 1, 1), (3, 256, 256), (1, 602, 256)):
        n = B.adaqp_orthogonalize_workspace_bytes(*sizes)
        assert n > 0 and n % 256 == 0
    assert B.adaqp_mx4_matmul_workspace_bytes(0, 5, 5) == 0 and B.adaqp_mx4_matmul_workspace_bytes(5, 5, 0) == 0
    assert B.adaqp_mx4_matmul_workspace_bytes(58_000, 256, 602) % 256 == 0
    L = B.lib()
    n = ctypes.c_int64()
    assert L.adaqp_layernorm_workspace_bytes(-1, 8, ctypes.byref(n)) == L.adaqp_layernorm_workspace_bytes(1, 0, ctypes.byref(n)) == B.EINVAL
    assert L.adaqp_layernorm_workspace_bytes(1, 8, None) == L.adaqp_mx4_matmul_workspace_bytes(1, 1, 1, None) == B.EINVAL
    assert L.adaqp_orthogonalize_workspace_bytes(1, 1, 1, None) == L.adaqp_orthogonalize_workspace_bytes(-1, 1, 1, ctypes.byref(n)) == B.EINVAL
    assert L.adaqp_mx4_matmul_workspace_bytes(1 << 31, 1, 1, ctypes.byref(n)) == B.ESIZE
    assert L.adaqp_orthogonalize_workspace_bytes(1, 1 << 20, 1, ctypes.byref(n)) == L.adaqp_orthogonalize_workspace_bytes(65536, 1, 1, ctypes.byref(n)) == B.ESIZE


def _refused(name, good, changes, **kw):
    """Each change of a good argument list is refused with its status; the good list itself is never called."""
    fn = getattr(B.lib(), name)
    for change, status in changes:
        args = list(good)
        for at, value in change.items():
            args[at] = value
        assert fn(*args) == status, (name, change)


def test_layernorm_refusals():
    forward = [P, 8, 4, 8, 0, P, P, 1e-5, P, 8, P, None]
    _refused("adaqp_layernorm_forward", forward, [
        ({0: None}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: 0}, B.EINVAL), ({4: 2}, B.EINVAL), ({4: -1}, B.EINVAL), ({5: P + 2}, B.EINVAL),
        ({6: P + 1}, B.EINVAL), ({7: -1.0}, B.EINVAL), ({7: float("nan")}, B.EINVAL), ({7: float("inf")}, B.EINVAL), ({8: None}, B.EINVAL), ({9: 7}, B.EINVAL),
        ({0: P + 2}, B.EINVAL), ({8: P + 1, 4: 1}, B.EINVAL), ({9: 9}, B.EINVAL), ({10: P + 2}, B.EINVAL)])
    assert B.lib().adaqp_layernorm_forward(None, 8, 0, 8, 0, None, None, 1e-5, None, 8, None, None) == B.OK
    backward = [P, 8, 2 * P, 8, 4, 8, 0, P, P, 3 * P, 8, P, P, P, 1 << 20, None]
    _refused("adaqp_layernorm_backward", backward, [
        ({0: None}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: None}, B.EINVAL), ({3: 7}, B.EINVAL), ({4: -1}, B.EINVAL), ({5: -8}, B.EINVAL), ({6: 5}, B.EINVAL),
        ({7: None}, B.EINVAL), ({10: 7}, B.EINVAL), ({11: None}, B.EINVAL), ({12: None}, B.EINVAL), ({13: None}, B.EINVAL), ({13: P + 16}, B.EINVAL),
        ({14: 255}, B.ESIZE), ({9: P, 10: 9}, B.EINVAL), ({9: 2 * P, 10: 9}, B.EINVAL), ({8: P + 1}, B.EINVAL)])
    assert B.lib().adaqp_layernorm_backward(P, 8, P, 8, 0, 8, 0, None, None, None, 8, None, None, None, 0, None) == B.OK


def test_mx4_refusals():
    good = [P, 8, 4, 8, 0, 0, 0, P, P, P, P, None]
    _refused("adaqp_mx4_quantize", good, [
        ({0: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({2: -1}, B.EINVAL), ({3: -1}, B.EINVAL), ({4: 3}, B.EINVAL), ({5: 2}, B.EINVAL),
        ({7: None}, B.EINVAL), ({8: None}, B.EINVAL), ({9: None}, B.EINVAL), ({10: None}, B.EINVAL), ({7: P + 4}, B.EINVAL), ({10: P + 8}, B.EINVAL),
        ({2: 1 << 31}, B.ESIZE), ({3: 1 << 31, 1: 1 << 31}, B.ESIZE)])
    assert B.lib().adaqp_mx4_quantize(None, 0, 0, 8, 0, 0, 0, None, None, None, None, None) == B.OK
    good = [P, P, 4, 8, P, 8, 0, None]
    _refused("adaqp_mx4_dequantize", good, [({0: None}, B.EINVAL), ({1: None}, B.EINVAL), ({1: P + 4}, B.EINVAL), ({2: -1}, B.EINVAL), ({4: None}, B.EINVAL),
                                            ({5: 7}, B.EINVAL), ({6: 9}, B.EINVAL), ({2: 1 << 31}, B.ESIZE)])
    good = [P, P, 4, P, P, 8, 16, P, 8, 0, P, 1 << 20, None]
    _refused("adaqp_mx4_matmul", good, [
        ({0: None}, B.EINVAL), ({1: None}, B.EINVAL), ({3: None}, B.EINVAL), ({4: P + 4}, B.EINVAL), ({2: -1}, B.EINVAL), ({5: -1}, B.EINVAL), ({6: -1}, B.EINVAL),
        ({7: None}, B.EINVAL), ({7: P + 2}, B.EINVAL), ({8: 7}, B.EINVAL), ({9: 2}, B.EINVAL), ({2: 1 << 31}, B.ESIZE), ({6: 1 << 31}, B.ESIZE)])
    need = B.adaqp_mx4_matmul_workspace_bytes(4, 8, 100_000)
    assert need > 0                                 # one tile: k is split
    _refused("adaqp_mx4_matmul", good, [({6: 100_000, 11: need - 1}, B.ESIZE), ({6: 100_000, 10: None}, B.EINVAL), ({6: 100_000, 10: P + 128}, B.EINVAL)])


def test_orthogonalize_refusals():
    coef = np.array(STEPS, dtype=np.float32)
    wild = np.array([[30.0, 0.0, 0.0]], dtype=np.float32)
    broken = np.array([[np.nan, 0.0, 0.0]], dtype=np.float32)
    good = [P, 8, 64, 2 * P, 8, 64, 2, 8, 8, 0, 5, coef.ctypes.data, 1e-7, P, 1 << 30, None]
    _refused("adaqp_orthogonalize", good, [
        ({0: None}, B.EINVAL), ({3: None}, B.EINVAL), ({0: P + 2}, B.EINVAL), ({1: 7}, B.EINVAL), ({4: 7}, B.EINVAL), ({2: 63}, B.EINVAL), ({5: 63}, B.EINVAL),
        ({6: -1}, B.EINVAL), ({7: -1}, B.EINVAL), ({8: -1}, B.EINVAL), ({9: 2}, B.EINVAL), ({10: -1}, B.EINVAL), ({10: 65}, B.ESIZE), ({11: None}, B.EINVAL),
        ({12: -1.0}, B.EINVAL), ({12: float("nan")}, B.EINVAL), ({13: None}, B.EINVAL), ({13: P + 4}, B.EINVAL), ({14: 1000}, B.ESIZE),
        ({10: 1, 11: wild.ctypes.data}, B.EINVAL), ({10: 1, 11: broken.ctypes.data}, B.EINVAL), ({7: 1 << 20, 2: 1 << 40, 5: 1 << 40}, B.ESIZE),
        ({3: P, 4: 9, 5: 80}, B.EINVAL)])
    assert B.lib().adaqp_orthogonalize(None, 0, 0, None, 0, 0, 0, 8, 8, 0, 5, coef.ctypes.data, 1e-7, None, 0, None) == B.OK


def test_random_numbers_are_those_of_the_codecs_generator(oracle):
    seed = 0x0123456789ABCDEF
    got = D.philox16(3, 24, seed)
    for row in range(3):
        for granule in range(3):
            words = oracle.philox4x32_10([granule, row, 0, D.MX_TAG], [seed & 0xFFFFFFFF, seed >> 32])
            want = [int(w) >> s & 0xFFFF for w in words for s in (0, 16)]
            assert got[row, 8 * granule:8 * granule + 8].tolist() == want


def test_mx4_definition_pins():
    """By hand: all 16 codes at scale 1, ties, a value beyond 6, zeros, the smallest scale."""
    v = np.concatenate([D.VALUES, -D.VALUES])
    x = np.zeros((1, 32))
    x[0, :16] = v
    codes, scales = D.mx4_quantize(x)
    assert scales.ravel().tolist() == [127, 0, 0, 0]
    assert codes[0, :8].tolist() == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] and not codes[0, 8:].any()
    assert np.array_equal(D.mx4_values(codes, scales, 32), x)
    x[0, :9] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7.9]                  # ties to the even code; 7.9 to 6
    codes, scales = D.mx4_quantize(x)
    assert scales[0, 0, 0] == 127 and D.mx4_values(codes, scales, 9)[0].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6]
    codes, scales = D.mx4_quantize(np.full((1, 40), 2.0 ** -140))
    assert scales[0, 0, :2].tolist() == [0, 0] and not (codes & 0x77).any()
    assert D.mx4_quantize(np.array([[6.0]]), seed=1)[1][0, 0, 0] == 127 and D.mx4_quantize(np.array([[6.1]]), seed=1)[1][0, 0, 0] == 128


def test_stochastic_rounding_is_unbiased_and_never_clips():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 64))
    got = np.stack([D.mx4_values(*D.mx4_quantize(x, seed), 64) for seed in range(4000)])
    step = got.max(0) - got.min(0)
    assert np.all(np.abs(got.mean(0) - x) <= 4 * step / np.sqrt(4 * 4000) + step * 2.0 ** -16)
    assert np.all(got.max(0) >= x) and np.all(got.min(0) <= x)


def test_orthogonalize_definition_is_the_polynomial_of_the_singular_values():
    rng = np.random.default_rng(1)
    for shape in ((5, 9), (9, 5), (1, 4), (6, 6)):
        g = rng.standard_normal(shape)
        u, s, vt = np.linalg.svd(g, full_matrices=False)
        s = s / np.sqrt((s * s).sum())
        for a, b, c in STEPS:
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(D.orthogonalize(g, STEPS, 0.0), u * s @ vt, atol=1e-12)


def test_layernorm_refuses_more_columns_than_it_counts():
    L, n = B.lib(), ctypes.c_int64()
    many = (1 << 30) + 1
    assert L.adaqp_layernorm_workspace_bytes(1, many, ctypes.byref(n)) == B.ESIZE
    assert L.adaqp_layernorm_forward(P, many, 1, many, 0, None, None, 1e-5, P, many, None, None) == B.ESIZE
    assert L.adaqp_layernorm_backward(P, many, 2 * P, many, 1, many, 0, P, None, 3 * P, many, None, None, None, 0, None) == B.ESIZE


def test_wrappers_refuse_tensors_that_are_not_what_they_name():
    """Found by the binding, before the library is asked."""
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.adaqp_layernorm_forward(x, 8, None, None, 1e-5, x)         # not on a device
    with pytest.raises(TypeError):
        B.adaqp_mx4_quantize(x, 8, B.MX4_NEAREST, 0, None, None)
    with pytest.raises(TypeError):
        B.adaqp_orthogonalize(x, x, STEPS, 1e-7, None)
    with pytest.raises(ValueError):
        B._same("call", (3, 0), (4, 0))


def test_stochastic_definition_holds_what_fp32_has():
    """2^128 = 4 * 2^126 is never written; below, magnitudes of such a block are rounded as in any other."""
    x = np.full((1, 32), 2.0 ** 128 * (1 - 2.0 ** -24))
    x[0, 1:4] = [-x[0, 0], 1.25 * 2.0 ** 126, 0.5 * 2.0 ** 126]
    seen = set()
    for seed in range(64):
        codes, scales = D.mx4_quantize(x, seed)
        assert scales.ravel().tolist() == [253, 0, 0, 0]
        v = D.mx4_values(codes, scales, 32)[0]
        assert v[0] == 3 * 2.0 ** 126 == -v[1] and np.all(v[4:] == v[0]) and v[3] == 0.5 * 2.0 ** 126
        seen.add(v[2] / 2.0 ** 126)
    assert seen == {1.0, 1.5}
    y = np.full((1, 32), 1.5 * 2.0 ** 127)                                    # the largest that the scale below holds
    codes, scales = D.mx4_quantize(y, 3)
    assert scales.ravel()[0] == 252 and np.array_equal(D.mx4_values(codes, scales, 32), y)


def test_workspace_of_updates_in_one_launch_is_that_of_their_norms():
    """Matrices that fit a CU's LDS need no memory for their steps; without steps their norms' partial sums: at most 512 of 8 bytes each."""
    for count, rows, cols in ((1000, 64, 64), (65535, 64, 64), (3, 41, 256), (7, 256, 41), (1, 1, 1)):
        need = B.adaqp_orthogonalize_workspace_bytes(count, rows, cols)
        assert need % 256 == 0 and 0 < need <= count * 512 * 8
    assert B.adaqp_orthogonalize_workspace_bytes(1, 65, 65) > 4 * 65 * 65 * 4


def test_layernorm_definition_has_the_gradients_of_differences():
    """Slopes of sum(dy * y) along random directions of x, gamma and beta.  Central differences of 1e-5 are off by 1e-10 of third derivatives (about 1 here) and by 1e-11 of the sum's size: 1e-7
    leaves room for both."""
    rng = np.random.default_rng(11)
    for rows, dim in ((1, 2), (5, 12), (20, 37)):
        x, dy, gamma, beta = 2 * rng.standard_normal((rows, dim)) + 0.5, rng.standard_normal((rows, dim)), rng.standard_normal(dim), rng.standard_normal(dim)
        eps, t = 1e-2, 1e-5
        _, mean, rstd = D.layernorm(x, gamma, beta, eps)
        dx, dgamma, dbeta = D.layernorm_backward(x, dy, mean, rstd, gamma)

        def loss(x, gamma, beta):
            return (dy * D.layernorm(x, gamma, beta, eps)[0]).sum()
        for _ in range(4):
            vx, vg, vb = rng.standard_normal((rows, dim)), rng.standard_normal(dim), rng.standard_normal(dim)
            slope = (loss(x + t * vx, gamma + t * vg, beta + t * vb) - loss(x - t * vx, gamma - t * vg, beta - t * vb)) / (2 * t)
            parts = [dx * vx, dgamma * vg, dbeta * vb]
            assert abs(sum(p.sum() for p in parts) - slope) <= 1e-7 * (1 + sum(np.abs(p).sum() for p in parts))


def test_mx4_definition_is_a_search_of_the_grid():
    """Of random blocks: the power of two by its inequality, and no value of the grid nearer than the one that the code stands for, at ties an even code."""
    rng = np.random.default_rng(12)
    x = rng.standard_normal((40, 96)) * np.exp2(rng.integers(-9, 10, size=(40, 3)).repeat(32, 1))
    x[::4] = np.round(x[::4] * 4) / 4                                         # ties among them
    x[5, 32:64] = 0.0
    grid = [float(v) for v in D.VALUES]
    codes, scales = D.mx4_quantize(x)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(40, -1)[:, :96]
    exponent = scales.transpose(1, 0, 2).reshape(40, -1)[:, :3].astype(int) - 127
    _, upper = D.mx4_quantize(x, seed=9)
    upper = upper.transpose(1, 0, 2).reshape(40, -1)[:, :3].astype(int) - 127
    for r in range(40):
        for b in range(3):
            block, e, s = x[r, 32 * b:32 * b + 32], exponent[r, b], upper[r, b]
            most = max(abs(v) for v in block)
            if most == 0.0:
                assert e == s == -127
                continue
            assert 4.0 * 2.0 ** e <= most < 8.0 * 2.0 ** e
            assert 6.0 * 2.0 ** (s - 1) < most <= 6.0 * 2.0 ** s
            for v, c in zip(block, code[r, 32 * b:32 * b + 32]):
                far = [abs(abs(v) / 2.0 ** e - g) for g in grid]
                assert far[c % 8] == min(far) and (far.count(min(far)) == 1 or c % 2 == 0)
                assert (c >= 8) == (np.signbit(v))


def test_wrappers_say_that_whole_lines_are_written():
    """Outputs may be views: each wrapper that writes a matrix says what becomes of the columns behind it."""
    for name in ("adaqp_layernorm_forward", "adaqp_layernorm_backward", "adaqp_mx4_dequantize", "adaqp_mx4_matmul", "adaqp_orthogonalize"):
        assert "128-byte lines" in getattr(B, name).__doc__, name


def test_the_updates_steps_do_what_their_comment_says():
    from paper_2306_01381_amd.dense import UPDATE_STEPS
    s = np.linspace(0.01, 1.0, 200_001)
    for a, b, c in UPDATE_STEPS:
        s = a * s + b * s ** 3 + c * s ** 5
    assert 0.68 <= s.min() < 0.69 and 1.13 < s.max() <= 1.14
