"""Layer norm on the GPU against the float64 oracle.

Tolerances, element by element, from the arithmetic (u = 2^-24, half a step of the
output type added): a row's mean is a sum in which no value passes more than 16
additions of its lane, 6 of its wave and 16 of the row's waves, so its error is
below 40 u mean|x|; a deviation adds u |x - mu|, and the variance (a sum of squares
of those, taken the same way) and its root cost less than 40 u of themselves. With
K = 64 this bounds xh by K u s, s = |xh| + r mean|x|, and y by K u s |w| plus a
rounding of the result. The backward's two row means pass as many additions, over
terms |u| and |u| s. The parameters' gradients add T terms |gy| s in lanes, blocks
and groups: no term passes more than 64 additions at the sizes here plus those of
xh (at most 40 rounds of a block's rows, 8 groups, 32 parts and 16 rows of them in
the largest ones), so 2 K u sum |gy| s.
"""

import numpy as np
import pytest
import torch

from oracle import post as P
from paper_2608_09703_amd import api as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
K = 64.0
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _np(x):
    return x.detach().double().cpu().numpy()


def _draw(T, d, act, par, seed, offset=0.5, bias=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(T, d, generator=g, device=DEV) * torch.exp(torch.randn(T, 1, generator=g, device=DEV))
         + offset).to(act)
    w = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(par)
    b = torch.randn(d, generator=g, device=DEV).to(par) if bias else None
    gy = torch.randn(T, d, generator=g, device=DEV).to(act)
    return x, w, b, gy


def _within(got, ref, bound, dtype, what):
    bad = ~(np.abs(got - ref) <= HALF[dtype] * np.abs(ref) + bound)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {ref[bad][0]}")


def _check(x, w, b, gy, eps, got, what):
    y, gx, gw, gb = got
    xn, wn, gn = _np(x), _np(w), _np(gy)
    bn = _np(b) if b is not None else np.zeros_like(wn)
    mu = xn.mean(1, keepdims=True)
    r = 1 / np.sqrt(((xn - mu) ** 2).mean(1, keepdims=True) + eps)
    s = np.abs(xn - mu) * r + r * np.abs(xn).mean(1, keepdims=True)
    ref = P.layer_norm(xn, wn, bn, eps)
    _within(_np(y), ref, K * U * (s * np.abs(wn) + np.abs(bn)), x.dtype, what + " y")
    rx, rw, rb = P.layer_norm_backward(xn, wn, gn, eps)
    au = np.abs(gn * wn)
    if gx is not None:
        bound = 2 * K * U * r * (au + au.mean(1, keepdims=True) + s * (au * s).mean(1, keepdims=True))
        _within(_np(gx), rx, bound, x.dtype, what + " gx")
    if gw is not None:
        _within(_np(gw), rw, 2 * K * U * (np.abs(gn) * s).sum(0), w.dtype, what + " gw")
    if gb is not None:
        _within(_np(gb), rb, 2 * K * U * np.abs(gn).sum(0), w.dtype, what + " gb")


def _run(x, w, b, gy, eps=1e-5):
    y, stats = D.layer_norm_forward(x, w, b, eps=eps, want_stats=True)
    return (y, *D.layer_norm_backward(x, w, stats, gy, eps=eps, want_bias=b is not None))


# widths at and around the edges of a lane's chunks, a wave, several waves; odd ones
WIDTHS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 504, 512, 513, 520, 1000, 1001, 1024, 1032, 2304, 4352, 4353, 8192, 8200,
          16383, 16384]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("act,par", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                     (torch.float32, torch.float32), (torch.float32, torch.bfloat16)])
def test_widths_and_types(d, act, par):
    T = 5
    x, w, b, gy = _draw(T, d, act, par, d)
    _check(x, w, b, gy, 1e-5, _run(x, w, b, gy), f"d={d}")


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 127, 512, 513, 1025, 3000, 8200])
@pytest.mark.parametrize("d", [40, 600, 1100, 2500])
@pytest.mark.parametrize("act", [torch.bfloat16, torch.float32])
def test_rows(T, d, act):
    """Fewer rows than blocks, one more than a round of blocks, several rounds of one and of two rows."""
    x, w, b, gy = _draw(T, d, act, torch.float32, T)
    _check(x, w, b, gy, 1e-5, _run(x, w, b, gy), f"T={T} d={d}")


@pytest.mark.parametrize("T,d,act", [(25000, 1500, torch.bfloat16), (70000, 500, torch.bfloat16), (9000, 4352,
                                     torch.bfloat16), (13000, 1303, torch.float32), (7000, 3001, torch.float32)])
def test_large_arrays(T, d, act):
    """Arrays of 64 MiB and more (streamed past the caches), where the sums over rows are long.
    No value passes more additions than its block has rounds (below 40), 8 groups, 32 parts and 16 rows."""
    x, w, b, gy = _draw(T, d, act, torch.bfloat16, d)
    assert x.numel() * x.element_size() >= 64 << 20
    _check(x, w, b, gy, 1e-5, _run(x, w, b, gy), f"T={T} d={d}")


@pytest.mark.parametrize("act", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,ld,off", [(64, 200, 0), (64, 200, 8), (64, 201, 1), (1000, 1008, 3), (1024, 4352, 1024)])
def test_columns_of_a_wider_array(act, d, ld, off):
    g = torch.Generator(device=DEV).manual_seed(d + off)
    wide = torch.randn(37, ld + off, generator=g, device=DEV).to(act)[:, off:]
    x = wide[:, :d]
    assert x.stride(0) == ld + off
    _, w, b, gy = _draw(37, d, act, torch.float32, 3)
    _check(x, w, b, gy, 1e-5, _run(x, w, b, gy), f"d={d} of {ld}")
    # 3-D rows of one distance
    x3 = torch.randn(4, 9, ld, generator=g, device=DEV).to(act)[:, :, :d]
    gy3 = torch.randn(x3.shape, generator=g, device=DEV).to(act)
    y, gx, gw, gb = _run(x3, w, b, gy3)
    assert y.shape == gx.shape == x3.shape
    assert torch.equal(y, D.layer_norm(x3.contiguous(), w, b))
    _check(x3.reshape(36, d), w, b, gy3.view(36, d), 1e-5, (y.view(36, d), gx.view(36, d), gw, gb), "3-D")


@pytest.mark.parametrize("off", [1, 4])
def test_unaligned_addresses(off):
    d = 512
    x, w, b, gy = _draw(9, d, torch.bfloat16, torch.bfloat16, 1)

    def shifted(t):
        buf = torch.empty(t.numel() + off, dtype=t.dtype, device=DEV)[off:].view(t.shape)
        return buf.copy_(t)
    ref = _run(x, w, b, gy)
    got = _run(shifted(x), shifted(w), shifted(b), shifted(gy))
    _check(x, w, b, gy, 1e-5, got, "unaligned")
    _check(x, w, b, gy, 1e-5, ref, "aligned")
    # an address does not change what is computed: the same bits
    for a, c in zip(ref, got):
        assert torch.equal(a, c)


@pytest.mark.parametrize("offset,eps", [(1000.0, 1e-5), (0.0, 10.0), (0.0, 1e-12)])
def test_offsets_and_eps(offset, eps):
    x, w, b, gy = _draw(33, 777, torch.float32, torch.float32, 5, offset=offset)
    _check(x, w, b, gy, eps, _run(x, w, b, gy, eps), f"offset {offset} eps {eps}")


def test_constant_and_non_finite_rows_stay_their_own():
    x, w, b, gy = _draw(6, 300, torch.float32, torch.float32, 6)
    ref = _run(x, w, b, gy)
    x = x.clone()
    x[1] = 3.0
    x[3, 7] = float("inf")
    x[4, 8] = float("nan")
    y, gx, _, _ = _run(x, w, b, gy)
    assert torch.equal(y[1], b) and torch.isfinite(gx[1]).all()
    assert torch.isnan(y[3]).any() and torch.isnan(y[4]).all()
    for k in (0, 2, 5):
        assert torch.equal(y[k], ref[0][k]) and torch.equal(gx[k], ref[1][k])


def test_each_output_alone_has_the_same_bits():
    x, w, b, gy = _draw(700, 520, torch.bfloat16, torch.float32, 7)
    y, stats = D.layer_norm_forward(x, w, b, want_stats=True)
    assert torch.equal(y, D.layer_norm_forward(x, w, b))
    full = D.layer_norm_backward(x, w, stats, gy, want_bias=True)
    for k, name in enumerate(("want_x", "want_weight", "want_bias")):
        only = {"want_x": False, "want_weight": False, "want_bias": False, name: True}
        got = D.layer_norm_backward(x, w, stats, gy, **only)
        assert torch.equal(got[k], full[k]) and [g is None for g in got].count(True) == 2
    again = D.layer_norm_backward(x, w, stats, gy, want_bias=True)
    assert all(torch.equal(a, c) for a, c in zip(full, again))


@pytest.mark.parametrize("bias", [True, False])
def test_autograd(bias):
    x, w, b, gy = _draw(20, 136, torch.bfloat16, torch.float32, 8, bias=bias)
    leaves = [t.requires_grad_(True) for t in (x, w, b) if t is not None]
    y = D.layer_norm(*leaves)
    y.backward(gy.t().contiguous().t())  # a gradient whose rows are not neighbours
    grads = [t.grad for t in leaves] + ([] if bias else [None])
    _check(x, w, b, gy, 1e-5, (y, *grads), "autograd")
    # frozen parameters
    x2 = x.detach().requires_grad_(True)
    D.layer_norm(x2, w.detach(), None if b is None else b.detach()).backward(gy)
    assert torch.equal(x2.grad, x.grad)
    with torch.no_grad():
        assert not D.layer_norm(*leaves).requires_grad


def test_refusals():
    x, w, b, _ = _draw(4, 64, torch.bfloat16, torch.float32, 9)
    for bad in (x.t(), x[:, ::2], x[:1].expand(4, 64), torch.empty(0, 64, device=DEV),
                torch.randn(3, 4, 64, device=DEV).transpose(0, 1)):
        with pytest.raises(ValueError):
            D.layer_norm(bad, torch.ones(bad.shape[-1], device=DEV))
    with pytest.raises(ValueError):
        D.layer_norm(x, w[:32])
    with pytest.raises(ValueError):
        D.layer_norm(x, w, b.bfloat16())
    with pytest.raises(TypeError):
        D.layer_norm(x.half(), w)
    with pytest.raises(RuntimeError):
        D.layer_norm(x, w.cpu())
    _, stats = D.layer_norm_forward(x, w, b, want_stats=True)
    for gy in (x.float(), x[:2], x.t().contiguous().t()):
        with pytest.raises(ValueError):
            D.layer_norm_backward(x, w, stats, gy)
    with pytest.raises(ValueError):
        D.layer_norm_backward(x, w, stats[:, :3], x)
