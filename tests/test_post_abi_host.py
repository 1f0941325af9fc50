"""Refusals of the post-training entry points. Everything is decided on the host before
any device call, so the addresses here are made up and never read."""

import ctypes
import math
import os

import pytest
import torch

from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B
from tests.test_abi_host import test_struct_layout_matches_header as _check_layout

A = 1 << 40  # fake, aligned addresses far apart


def _at(i, off=0):
    return A + (i << 34) + off


@pytest.mark.parametrize("cname,cls", [("mls_layer_norm", B.LayerNorm), ("mls_policy", B.Policy),
                                       ("mls_grad_tensor", B.GradTensor)])
def test_struct_layouts_match_the_header(tmp_path, cname, cls):
    _check_layout(tmp_path, cname, cls)


def _refused(status, call, *args, text=None):
    with pytest.raises(B.MlsError) as e:
        call(*args)
    assert e.value.status == status, e.value
    if text:
        assert text in str(e.value)


# -- layer norm ----------------------------------------------------------------

def _norm(T=8, d=64, ld=None, act=B.MLS_BF16, par=B.MLS_F32, eps=1e-5):
    return B.make_layer_norm(T, d, d if ld is None else ld, act, par, eps)


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), B.MLS_INVALID_ARG), (dict(d=0), B.MLS_UNSUPPORTED), (dict(d=16385), B.MLS_UNSUPPORTED),
    (dict(ld=63), B.MLS_INVALID_ARG), (dict(act=2), B.MLS_UNSUPPORTED), (dict(par=-1), B.MLS_UNSUPPORTED),
    (dict(eps=0.0), B.MLS_INVALID_ARG), (dict(eps=-1.0), B.MLS_INVALID_ARG),
    (dict(eps=math.nan), B.MLS_INVALID_ARG), (dict(eps=math.inf), B.MLS_INVALID_ARG)])
def test_layer_norm_descriptors(kw, status):
    n = _norm(**kw)
    _refused(status, B.layer_norm_workspace, n)
    _refused(status, B.layer_norm_fwd, n, _at(1), _at(2), None, _at(3), None, None)
    _refused(status, B.layer_norm_bwd, n, _at(1), _at(2), _at(3), _at(4), _at(5), None, None, None, 0, None)


def test_layer_norm_pointers():
    n = _norm()
    fwd = lambda x=_at(1), w=_at(2), b=None, y=_at(3), st=None: B.layer_norm_fwd(n, x, w, b, y, st, None)  # noqa: E731
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(x=_at(1, 1)), dict(y=_at(3, 1)), dict(w=_at(2, 2)),
               dict(b=_at(4, 2)), dict(st=_at(4, 2)), dict(y=_at(1)), dict(y=_at(1, 8 * 64 * 2 - 2))):
        _refused(B.MLS_INVALID_ARG, lambda: fwd(**kw))

    def bwd(x=_at(1), w=_at(2), st=_at(3), gy=_at(4), gx=_at(5), gw=None, gb=None, ws=_at(8), nb=1 << 30):
        B.layer_norm_bwd(n, x, w, st, gy, gx, gw, gb, ws, nb, None)
    for kw in (dict(x=None), dict(w=None), dict(st=None), dict(gy=None), dict(gx=_at(5, 1)), dict(gw=_at(6, 2)),
               dict(gb=_at(7, 2)), dict(ws=_at(8, 4), gw=_at(6)), dict(gx=_at(1)), dict(gx=_at(4))):
        _refused(B.MLS_INVALID_ARG, lambda: bwd(**kw))
    need = B.layer_norm_workspace(n)
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: bwd(gw=_at(6), nb=need - 1))
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: bwd(gb=_at(6), ws=None))
    bwd(gx=None)  # nothing asked for: nothing is enqueued


def test_layer_norm_workspace_does_not_grow_without_bound():
    for d in (1, 100, 4352, 16384):
        sizes = [B.layer_norm_workspace(_norm(T=T, d=d)) for T in (1, 7, 512, 5000, 1 << 20, 1 << 31)]
        assert sizes == sorted(sizes) and sizes[-1] == sizes[-2] and sizes[0] >= 8 * d


# -- token log-probabilities -----------------------------------------------------

def _problem(**kw):
    M = kw.pop("M", 1)
    return B.make_problem(M, kw.pop("T", 300), kw.pop("V", 5000), [kw.pop("d", 64)] * M, [_at(1)] * M,
                          [_at(2)] * M, _at(3), **kw)


def test_token_logp_refusals():
    p = _problem()
    ws, wb, kb = B.token_logp_workspace(p)
    assert kb >= 384 * 5120 * 2
    fwd = lambda q=p, s=_at(4), lp=_at(5), en=None, k=None, w=_at(6), nb=ws: B.token_logp_fwd(q, s, lp, en, k, w, nb, None)  # noqa: E731
    bwd = lambda q=p, s=_at(4), g=_at(5), gh=_at(7), gW=_at(8), k=None, w=_at(6), nb=wb: B.token_logp_bwd(  # noqa: E731
        q, s, k, g, gh, gW, w, nb, None)
    for call in (fwd, bwd):
        _refused(B.MLS_INVALID_ARG, lambda: call(q=_problem(M=2)), text="one sub-model")
        _refused(B.MLS_INVALID_ARG, lambda: call(q=_problem(tau=0.0)))
        _refused(B.MLS_INVALID_ARG, lambda: call(q=_problem(tau=math.nan)))
        _refused(B.MLS_INVALID_ARG, lambda: call(q=_problem(T=0)))
        _refused(B.MLS_INVALID_ARG, lambda: call(q=_problem(V=1)))
        _refused(B.MLS_UNSUPPORTED, lambda: call(q=_problem(d=60)))
        _refused(B.MLS_UNSUPPORTED, lambda: call(q=_problem(dtype=5)))
        for kw in (dict(s=None), dict(w=None), dict(s=_at(4, 8)), dict(w=_at(6, 8))):
            _refused(B.MLS_INVALID_ARG, lambda: call(**kw))
        _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: call(nb=16))
        _refused(B.MLS_INVALID_ARG, lambda: call(k=_at(9, 8)))
        f32 = _problem(dtype=B.MLS_F32)
        assert B.token_logp_workspace(f32)[2] == 0
        _refused(B.MLS_UNSUPPORTED, lambda: call(q=f32, k=_at(9), nb=1 << 40), text="kept")
    for kw in (dict(lp=None), dict(lp=_at(5, 2)), dict(en=_at(9, 1))):
        _refused(B.MLS_INVALID_ARG, lambda: fwd(**kw))
    for kw in (dict(g=None), dict(g=_at(5, 2)), dict(gh=_at(7, 2)), dict(gW=_at(8, 2))):
        _refused(B.MLS_INVALID_ARG, lambda: bwd(**kw))


def test_a_token_logp_workspace_for_the_longest_batch_serves_the_shorter_ones():
    last = (0, 0, 0)
    for T in (1, 127, 128, 129, 300, 512, 1000, 2000, 4096, 9000):
        now = B.token_logp_workspace(_problem(T=T, V=50000, d=512, grad_h_dtype=B.MLS_BF16))
        assert all(a >= b for a, b in zip(now, last))
        assert now[0] < T * 50000 * 4 // 2 + (1 << 26)
        last = now


# -- policy loss -----------------------------------------------------------------

@pytest.mark.parametrize("kw", [
    dict(N=0), dict(N=1 << 31), dict(S=-1), dict(flags=4, S=1), dict(flags=1), dict(flags=2),
    dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_low=math.nan), dict(clip_high=-0.1),
    dict(clip_high=math.nan), dict(kl_coef=-1.0), dict(kl_coef=math.inf), dict(kl_coef=math.nan)])
def test_policy_descriptors(kw):
    kw = {"N": 10, **kw}
    p = B.make_policy(**kw)
    _refused(B.MLS_INVALID_ARG, B.policy_loss_workspace, p)


def test_policy_pointers():
    p = B.make_policy(10, 2, flags=B.MLS_POLICY_MEAN_OF_SEQUENCES, clip_high=math.inf)
    nb = B.policy_loss_workspace(p)

    def fwd(q=p, lp=_at(1), old=_at(2), adv=_at(3), ref=None, mask=None, cu=_at(4), loss=_at(5), kl=None, cl=None,
            grad=None, ws=_at(6), n=nb):
        B.policy_loss_fwd(q, lp, old, adv, ref, mask, cu, loss, kl, cl, grad, ws, n, None)
    for kw in (dict(lp=None), dict(old=None), dict(adv=None), dict(loss=None), dict(ws=None), dict(cu=None),
               dict(q=B.make_policy(10)), dict(q=B.make_policy(10, 2, kl_coef=0.1)), dict(lp=_at(1, 2)),
               dict(ref=_at(7, 2)), dict(cu=_at(4, 2)), dict(grad=_at(7, 1)), dict(kl=_at(7, 1)),
               dict(cl=_at(7, 2)), dict(ws=_at(6, 8))):
        _refused(B.MLS_INVALID_ARG, lambda: fwd(**kw))
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: fwd(n=nb - 1))
    for args in ((0, _at(1), _at(2), _at(3)), (5, None, _at(2), _at(3)), (5, _at(1), None, _at(3)),
                 (5, _at(1), _at(2), None), (5, _at(1, 2), _at(2), _at(3))):
        _refused(B.MLS_INVALID_ARG, B.policy_loss_bwd, *args, None)


# -- gradient clipping -----------------------------------------------------------

def _clip(rows, max_norm=1.0, norm=_at(100), ws=_at(101), nb=None):
    t = B.make_grad_tensors(*zip(*rows))
    B.clip_grad_norm(len(rows), t, max_norm, norm, ws, (1 << 30) if nb is None else nb, None)


def test_clip_refusals():
    ok = (_at(1), _at(1), 100, B.MLS_F32)
    bad = [(_at(1), _at(1), 100, 3), (_at(1), _at(1), -1, B.MLS_F32), (None or 0, _at(1), 100, B.MLS_F32),
           (_at(1), 0, 100, B.MLS_F32), (_at(1, 2), _at(1, 2), 100, B.MLS_F32), (_at(1, 1), _at(1, 1), 9, B.MLS_BF16),
           (_at(1), _at(1, 4), 100, B.MLS_F32), (_at(1), _at(1), (1 << 40) + 1, B.MLS_F32),
           (_at(1), _at(1), 100, B.MLS_F32 | (1 << 32))]
    for row in bad:
        with pytest.raises(B.MlsError):
            _clip([(_at(2), _at(2), 10, B.MLS_BF16), row])
    for kw in (dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(ws=None), dict(norm=_at(100, 2)),
               dict(ws=_at(101, 4))):
        _refused(B.MLS_INVALID_ARG, lambda: _clip([ok], **kw))
    t = B.make_grad_tensors(*zip(ok))
    need = B.clip_grad_norm_workspace(1, t)
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: _clip([ok], nb=need - 1))


@pytest.mark.parametrize("rows", [
    # the same gradient twice; two outputs in one place; an output on another input; one that ends inside another
    [(_at(1), _at(1), 10, 1), (_at(1), _at(1), 10, 1)],
    [(_at(1), _at(3), 10, 1), (_at(2), _at(3), 10, 1)],
    [(_at(1), _at(2), 10, 1), (_at(2), _at(3), 10, 1)],
    [(_at(1), _at(3), 10, 1), (_at(2), _at(3, 36), 10, 0)],
    [(_at(1), _at(1), 1000, 1), (_at(2), _at(2), 10, 1), (_at(1, 400), _at(3), 10, 1)]])
def test_clip_outputs_that_overlap(rows):
    _refused(B.MLS_INVALID_ARG, lambda: _clip(rows), text="overlaps")
    _refused(B.MLS_INVALID_ARG, lambda: _clip(rows[::-1]), text="overlaps")


def test_clip_workspace_follows_the_launches():
    def need(*sizes):
        return B.clip_grad_norm_workspace(len(sizes), B.make_grad_tensors([_at(1)] * len(sizes), [_at(1)] * len(sizes), sizes, [0] * len(sizes)))
    assert need() == need(0, 0) <= 512
    assert need(1) <= need(1 << 20) <= need(1 << 30) <= 2048 * 8 + 512
    assert need(*[1] * 500) <= 500 * 8 + 512


# -- the front end's own checks -----------------------------------------------------

def test_front_end_refuses_before_the_library():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(RuntimeError):
        D.layer_norm(x, w)
    with pytest.raises(RuntimeError):
        D.token_logp(x, torch.zeros(9, 8), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(RuntimeError):
        D.policy_loss(torch.zeros(4), torch.zeros(4), torch.zeros(4))
    with pytest.raises(RuntimeError):
        D.clip_grad_norm([x], 1.0)
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError):
            D.clip_grad_norm([x], bad)
    with pytest.raises(ValueError):
        D.clip_grad_norm([], 1.0)
    with pytest.raises(ValueError):
        D.grad_norm([None])


def test_every_entry_point_is_declared():
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mls.h")).read()
    for n in ("mls_layer_norm_fwd", "mls_token_logp_bwd", "mls_policy_loss_fwd", "mls_clip_grad_norm"):
        assert f"mls_status {n}(" in src and hasattr(B.lib(), n)
    assert ctypes.sizeof(B.GradTensor) == 32
