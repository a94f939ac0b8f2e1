"""The gradient of rotary positions against differences of the operation, element by element.

A step h in one column of a pair moves that pair's two outputs and no others, so a step in all first (or all second) columns at once
gives every element of the gradient: (g . (y(x + h) - y(x))) / h over the pair.  Each y is off by its own tolerance (test_rope_gpu.py),
the gradient by its own; with |x| < 4 in steps of 1/16 and h = 4, x + h is exact in bf16 and the bound about a fiftieth of the gradient."""
import numpy as np
import pytest

from _kv_util import bf16, bf16_cuda, host
from test_rope_gpu import reference

H, SCALE, R = 4.0, 1.5, 48


def operands():
    rng = np.random.default_rng(12)
    x = np.clip(np.round(rng.standard_normal((2, 3, 5, 64)) * 16) / 16, -3.9375, 3.9375)
    positions = rng.integers(0, 5000, (2, 5)).astype(np.int32)
    inv = 10000.0 ** (-np.arange(0, R, 2) / R)
    return x, bf16(rng.standard_normal(x.shape)), positions, inv


def parts(interleaved):
    return (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))


def differences(x, g, positions, inv, interleaved, operation):
    """(part, quotient, its tolerance) for a step in the first and in the second columns."""
    first, second = parts(interleaved)
    y0, (_, t0) = operation(x), reference(x, positions, inv, interleaved, False, SCALE)
    for part in (first, second):
        moved = x.copy()
        moved[..., part] += H
        assert np.array_equal(bf16(moved), moved)
        y1, (_, t1) = operation(moved), reference(moved, positions, inv, interleaved, False, SCALE)
        both = lambda a: a[..., first] + a[..., second]
        yield part, both((y1 - y0) * g) / H, both((t0 + t1) * np.abs(g)) / H


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_bound_tells_a_wrong_gradient(interleaved):
    """In 64 bits, no GPU: the right gradient is within it, none, the other direction's and one without the scale are not."""
    x, g, positions, inv = operands()
    exact = lambda z: reference(z, positions, inv, interleaved, False, SCALE)[0]
    right, tol = reference(g, positions, inv, interleaved, True, SCALE)
    wrong = [np.zeros_like(g), reference(g, positions, inv, interleaved, False, SCALE)[0], reference(g, positions, inv, interleaved, True, 1.0)[0]]
    for part, got, slack in differences(x, g, positions, inv, interleaved, exact):
        bound = slack + tol[..., part]
        assert np.all(np.abs(got - right[..., part]) <= 1e-9)
        assert bound.mean() < 0.04 * np.abs(right[..., part]).mean()
        for other in wrong:
            assert np.mean(np.abs(got - other[..., part]) > bound) > 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_against_differences(interleaved):
    import torch
    from paper_2604_18616_amd import binding
    x, g, positions, inv = operands()
    pos, freq = torch.from_numpy(positions).cuda(), torch.from_numpy(inv).cuda()
    run = lambda z, inverse: host(binding.rope_bf16(bf16_cuda(z), pos, freq, interleaved=interleaved, inverse=inverse, scale=SCALE))
    grad, tol = run(g, True), reference(g, positions, inv, interleaved, True, SCALE)[1]
    for part, got, slack in differences(x, g, positions, inv, interleaved, lambda z: run(z, False)):
        assert np.all(np.abs(got - grad[..., part]) <= slack + tol[..., part])
    assert np.array_equal(grad[..., R:], g[..., R:])
