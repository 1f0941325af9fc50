"""Gradient norm and clipping on the GPU against the float64 oracle.

The norm is a 64-bit sum rounded to fp32: 2^-24 of itself (and 1e-12 for the sum). A
scaled value is an fp32 product with an fp32 coefficient, rounded to its type: 2^-8
(bf16) or 2^-24 (fp32) of itself, plus 2 * 2^-24 for the coefficient and the product.
"""

import numpy as np
import pytest
import torch

from oracle import post as P
from paper_2608_09703_amd import api as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _np(x):
    return x.detach().double().cpu().numpy()


def _draw(sizes, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n, generator=g, device=DEV) * scale).to(torch.bfloat16 if (i + seed) % 2 else torch.float32)
            for i, n in enumerate(sizes)]


def _check(grads, max_norm, out=None):
    before = [x.clone() for x in grads]
    norm, want = P.clip([_np(x) for x in before], max_norm)
    alone = D.grad_norm(grads)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    got = D.clip_grad_norm(grads, max_norm, out=out)
    assert got.shape == () and got.dtype == torch.float32 and torch.equal(got, alone)
    assert abs(float(got) - norm) <= (U + 1e-12) * norm
    if out is not None:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))
    for x, b, w in zip(grads if out is None else out, before, want):
        x = _np(x)
        assert np.all(np.abs(x - w) <= (HALF[b.dtype] + 2 * U) * np.abs(w) + 1e-45)
    return got


SIZES = [[1], [7], [8], [8191], [8192], [8193], [0, 5, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9], [100000, 1, 70000, 3],
         [16384, 8, 24577], [3] * 137, [5] * 193, [17] * 400 + [30000]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda v: f"{len(v)}x{sum(v)}")
@pytest.mark.parametrize("seed", [0, 1])
def test_sizes_and_types(sizes, seed):
    """Tiles that a tensor ends in, empty tensors, more tensors than a launch takes."""
    grads = _draw(sizes, seed)
    _check([x.clone() for x in grads], 0.5)
    _check([x.clone() for x in grads], 0.5, out=[torch.full_like(x, float("nan")) for x in grads])


@pytest.mark.parametrize("seed", [0, 1])
def test_below_the_limit_everything_stays(seed):
    grads = _draw([1000, 9000, 3], seed)
    before = [x.clone() for x in grads]
    _check(grads, 1e6)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    out = [torch.empty_like(x) for x in grads]
    D.clip_grad_norm(grads, 1e6, out=out)
    assert all(torch.equal(a, b) for a, b in zip(before, out))
    D.clip_grad_norm(grads, float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(before, grads))


@pytest.mark.parametrize("off", [1, 3, 4, 8])
def test_addresses_that_are_no_multiple_of_16_bytes(off):
    """Tensors of one flat buffer, and outputs aligned otherwise than their inputs."""
    sizes = [20001, 9, 8192, 33333]
    for dt in (torch.bfloat16, torch.float32):
        flat = torch.randn(sum(sizes) + off, device=DEV).to(dt)
        src, at = [], off
        for n in sizes:
            src.append(flat[at:at + n])
            at += n
        _check(src, 0.7, out=[torch.empty_like(x) for x in src])
        _check([x.clone() for x in src], 0.7, out=src)


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_squares_beyond_float32(scale):
    grads = [(torch.randn(5000, device=DEV) * scale).to(dt) for dt in (torch.float32, torch.bfloat16)]
    _check(grads, 1.0 if scale > 1 else 1e-30)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    grads = _draw([5000, 300], 0)
    grads[1][17] = bad
    before = [x.clone() for x in grads]
    norm = D.clip_grad_norm(grads, 0.1)
    assert not torch.isfinite(norm)
    assert all(torch.equal(a, b) for a, b in zip(before[:1], grads[:1]))
    assert torch.equal(before[1].nan_to_num(7, 7), grads[1].nan_to_num(7, 7))
    assert not torch.isfinite(D.grad_norm(grads))


def test_zero_gradients_and_entries_without_one():
    z = [torch.zeros(100, device=DEV), None, torch.zeros(9, dtype=torch.bfloat16, device=DEV)]
    assert float(D.clip_grad_norm(z, 1.0)) == 0.0 and not z[0].any()
    z[0][3] = 3.0
    assert float(D.grad_norm(z)) == 3.0


def test_shapes_and_repeats():
    """Parameters' shapes; the same bits on every call."""
    grads = [torch.randn(50, 70, device=DEV), torch.randn(3, 4, 5, device=DEV).bfloat16(), torch.randn((), device=DEV)]
    _check([x.clone() for x in grads], 0.3)
    a = [D.grad_norm(grads) for _ in range(3)]
    assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])


def test_refusals():
    x = torch.randn(64, 64, device=DEV)
    for bad in ([x.t()], [x[:, ::2]], [x.cpu(), x], [x, x.cpu()]):
        with pytest.raises((ValueError, RuntimeError)):
            D.clip_grad_norm(bad, 1.0)
    with pytest.raises(TypeError):
        D.clip_grad_norm([x.half()], 1.0)
    for out in ([x.bfloat16()], [x[:5]], [], [x.clone().t()]):
        with pytest.raises(ValueError):
            D.clip_grad_norm([x], 1.0, out=out)
    with pytest.raises(RuntimeError):  # listed twice: scaled twice
        D.clip_grad_norm([x, x], 1.0)
    assert abs(float(D.grad_norm([x, x])) - 2 ** 0.5 * float(x.double().norm())) < 1e-4  # a norm of both is fine
