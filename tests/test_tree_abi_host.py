"""Refusals of the entry points for decoding with a tree of drafted tokens. Everything is decided on the
host before any device call, so the addresses here are made up and never read."""

import math

import pytest
import torch

from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B
from tests.test_abi_host import test_struct_layout_matches_header as _check_layout

A = 1 << 40  # fake, aligned addresses far apart


def _at(i, off=0):
    return A + (i << 34) + off


def test_struct_layout(tmp_path):
    _check_layout(tmp_path, "mls_kv_cache", B.KVCache)


def _refused(status, call, *args, text=None):
    with pytest.raises(B.MlsError) as e:
        call(*args)
    assert e.value.status == status, e.value
    if text:
        assert text in str(e.value)


def _cache(**kw):
    D_, ps, H, P = kw.get("head_dim", 64), kw.get("page_size", 16), kw.get("kv_heads", 2), kw.get("pages", 9)
    f = dict(dtype=B.MLS_BF16, page_size=ps, kv_heads=H, head_dim=D_, layers=1, pages=P, batch=3, table_pages=4,
             ld_layer=P * H * ps * D_, ld_page=H * ps * D_, ld_head=ps * D_, ld_entry=D_, ld_table=4, k=_at(1), v=_at(2),
             page_table=_at(3), lengths=_at(4))
    f.update(kw)
    return B.KVCache(**f)


def _write(c, n=5, k=_at(5), v=_at(6), ld=(640, 128, 64), counts=None):
    B.cache_write(c, n, k, v, ld, counts, None)


def _compact(c, n=5, path=_at(5), acc=_at(6), new=_at(7)):
    B.cache_compact(c, n, path, acc, new, None)


def _attend(c, n=5, heads=4, q=_at(5), ld=(1280, 256, 64), parents=_at(6), scale=0.1, out=_at(7), ws=_at(8), nb=1 << 33):
    B.tree_attention(c, n, heads, q, ld, parents, scale, out, ws, nb, None)


BAD_CACHES = [
    (dict(dtype=2), B.MLS_UNSUPPORTED), (dict(page_size=8), B.MLS_UNSUPPORTED), (dict(page_size=24), B.MLS_UNSUPPORTED),
    (dict(page_size=1 << 17), B.MLS_UNSUPPORTED), (dict(kv_heads=0), B.MLS_INVALID_ARG),
    (dict(head_dim=0), B.MLS_UNSUPPORTED), (dict(head_dim=60), B.MLS_UNSUPPORTED), (dict(head_dim=2048), B.MLS_UNSUPPORTED),
    (dict(layers=0), B.MLS_INVALID_ARG), (dict(pages=0), B.MLS_INVALID_ARG), (dict(pages=1 << 31), B.MLS_INVALID_ARG),
    (dict(batch=0), B.MLS_INVALID_ARG), (dict(batch=65536), B.MLS_INVALID_ARG), (dict(table_pages=0), B.MLS_INVALID_ARG),
    (dict(table_pages=1 << 30, ld_table=1 << 30), B.MLS_INVALID_ARG), (dict(ld_table=3), B.MLS_INVALID_ARG),
    (dict(ld_page=-64), B.MLS_INVALID_ARG), (dict(ld_head=1028), B.MLS_INVALID_ARG), (dict(ld_entry=0), B.MLS_INVALID_ARG),
    (dict(ld_entry=56), B.MLS_INVALID_ARG), (dict(ld_page=0), B.MLS_INVALID_ARG), (dict(ld_entry=1 << 26), B.MLS_UNSUPPORTED),
    (dict(k=None), B.MLS_INVALID_ARG), (dict(v=None), B.MLS_INVALID_ARG), (dict(page_table=None), B.MLS_INVALID_ARG),
    (dict(lengths=None), B.MLS_INVALID_ARG), (dict(k=_at(1, 8)), B.MLS_INVALID_ARG), (dict(v=_at(2, 2)), B.MLS_INVALID_ARG),
    (dict(page_table=_at(3, 2)), B.MLS_INVALID_ARG), (dict(lengths=_at(4, 1)), B.MLS_INVALID_ARG)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches(kw, status):
    c = _cache(**kw)
    _refused(status, _write, c)
    _refused(status, _compact, c)
    _refused(status, _attend, c)
    _refused(status, B.tree_attention_workspace, c, 5, 4)


def test_several_layers_are_the_compactions_alone():
    c = _cache(layers=2)
    _refused(B.MLS_INVALID_ARG, _write, c)
    _refused(B.MLS_INVALID_ARG, _attend, c)
    _refused(B.MLS_INVALID_ARG, _compact, _cache(layers=1 << 17))
    _refused(B.MLS_INVALID_ARG, _compact, _cache(layers=2, ld_layer=0))


def test_write():
    c = _cache()
    for kw in (dict(n=0), dict(n=1 << 31), dict(k=None), dict(v=None), dict(k=_at(5, 8)), dict(v=_at(6, 4)),
               dict(ld=(640, 128, 60)), dict(ld=(-640, 128, 64)), dict(ld=(640, 4, 64)), dict(counts=_at(7, 2))):
        _refused(B.MLS_INVALID_ARG, lambda: _write(c, **kw))


def test_compact():
    c = _cache()
    _refused(B.MLS_UNSUPPORTED, lambda: _compact(c, n=0))
    _refused(B.MLS_UNSUPPORTED, lambda: _compact(c, n=65))
    for kw in (dict(path=None), dict(acc=None), dict(new=None), dict(path=_at(5, 2)), dict(new=_at(7, 1)),
               dict(new=_at(4)), dict(new=_at(4, 8)), dict(new=_at(6)), dict(new=_at(5, 16))):
        _refused(B.MLS_INVALID_ARG, lambda: _compact(c, **kw))


def test_attention():
    c = _cache()
    need = B.tree_attention_workspace(c, 5, 4)
    assert need == 0  # one part
    for n in (0, 65):
        _refused(B.MLS_UNSUPPORTED, lambda: _attend(c, n=n))
    for kw in (dict(heads=3), dict(heads=0), dict(q=None), dict(out=None), dict(q=_at(5, 2)), dict(out=_at(7, 8)),
               dict(parents=_at(6, 2)), dict(scale=math.nan), dict(scale=math.inf), dict(scale=0.0), dict(scale=-1.0),
               dict(ld=(1280, 250, 64))):
        _refused(B.MLS_INVALID_ARG, lambda: _attend(c, **kw))
    for d in (16, 48, 512):
        _refused(B.MLS_UNSUPPORTED, lambda: _attend(_cache(head_dim=d)))
    long = _cache(table_pages=4000, ld_table=4000)
    need = B.tree_attention_workspace(long, 5, 4)
    assert need >= 3 * 2 * 10 * 64 * 4
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: _attend(long, nb=need - 1))
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: _attend(long, ws=None))
    _refused(B.MLS_INVALID_ARG, lambda: _attend(long, ws=_at(8, 4)))
    _refused(B.MLS_UNSUPPORTED, lambda: _attend(
        _cache(batch=65535, kv_heads=1024, table_pages=1 << 20, ld_table=1 << 20), heads=1024))


def _verify(V=1000, T=0.7, top_p=0.9, greedy=False, batch=2, n=5, target=_at(1), draft=_at(2), tokens=_at(3), parents=_at(4),
            ua=_at(5), us=_at(6), acc=_at(7), path=_at(8), nxt=_at(9), ws=_at(10), nb=1 << 33, rec=None):
    B.tree_verify(B.make_sampling(V, T, top_p, greedy), batch, n, target, draft, tokens, parents, ua, us, acc, path, nxt,
                  ws, nb, None, draft_params=rec)


def test_verify():
    for kw in (dict(T=0.0), dict(T=math.nan), dict(top_p=0.0), dict(top_p=1.5), dict(batch=0), dict(n=0), dict(n=65),
               dict(batch=1 << 25), dict(target=None), dict(tokens=None), dict(acc=None), dict(path=None), dict(nxt=None),
               dict(ua=None), dict(us=None), dict(target=_at(1, 2)), dict(tokens=_at(3, 1)), dict(parents=_at(4, 2)),
               dict(path=_at(8, 2)), dict(ws=_at(10, 8)), dict(rec=_at(11), draft=None), dict(rec=_at(11, 2))):
        _refused(B.MLS_INVALID_ARG, lambda: _verify(**kw))
    for V in (1, 65537):
        _refused(B.MLS_UNSUPPORTED, lambda: _verify(V=V))
    s = B.make_sampling(1000, 0.7, 0.9, False)
    need = B.tree_verify_workspace(s, 2, 5)
    assert need >= 2 * 1000 * 28
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: _verify(nb=need - 1))
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: _verify(ws=None))
    assert B.tree_verify_workspace(B.make_sampling(1000, greedy=True), 2, 5) == 0
    _refused(B.MLS_INVALID_ARG, B.tree_verify_workspace, s, 0, 5)


def test_quantize_and_head():
    q = lambda T=4, d=32, ld=32, dt=B.MLS_BF16, x=_at(1), q=_at(2), s=_at(3): B.quantize_rows(T, d, ld, dt, x, q, s, None)  # noqa: E731
    for kw in (dict(T=0), dict(T=1 << 31), dict(d=0), dict(d=(1 << 17) + 1), dict(ld=31), dict(x=None), dict(q=None),
               dict(s=None), dict(x=_at(1, 1)), dict(s=_at(3, 2)), dict(q=_at(1)), dict(q=_at(1, 4 * 64 - 1)), dict(s=_at(1)),
               dict(s=_at(2, 4))):
        _refused(B.MLS_INVALID_ARG, lambda: q(**kw))
    _refused(B.MLS_UNSUPPORTED, lambda: q(dt=3))
    h = lambda T=4, V=9, d=32, dt=B.MLS_BF16, o=_at(1), W=_at(2), s=_at(3), out=_at(4), ws=_at(5), nb=1 << 33: B.head_logits_int8(T, V, d, dt, o, W, s, out, ws, nb, None)  # noqa: E731,E501
    for kw in (dict(T=0), dict(T=(1 << 30) + 1), dict(V=0), dict(o=None), dict(W=None), dict(s=None), dict(out=None),
               dict(o=_at(1, 8)), dict(W=_at(2, 4)), dict(out=_at(4, 4)), dict(s=_at(3, 2)), dict(ws=_at(5, 4))):
        _refused(B.MLS_INVALID_ARG, lambda: h(**kw))
    for kw in (dict(d=24), dict(dt=-1)):
        _refused(B.MLS_UNSUPPORTED, lambda: h(**kw))
    need = B.head_logits_int8_workspace(4, 32)
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: h(nb=need - 1))
    _refused(B.MLS_WORKSPACE_TOO_SMALL, lambda: h(ws=None))


# -- the PyTorch front end ---------------------------------------------------------

def test_front_end_refuses_tensors_on_the_host():
    x = torch.zeros(1, 1, 1, 64)
    pages = torch.zeros(2, 1, 16, 64)
    table, lengths = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: D.cache_write(x, x, pages, pages, table, lengths),
                 lambda: D.cache_compact(pages, pages, table, lengths, table, lengths),
                 lambda: D.tree_attention(x, pages, pages, table, lengths),
                 lambda: D.tree_verify(torch.zeros(1, 2, 5), table, None, None, None, greedy=True),
                 lambda: D.quantize_rows(torch.zeros(2, 16)),
                 lambda: D.head_logits_int8(torch.zeros(1, 16), torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3))):
        with pytest.raises(RuntimeError, match="GPU only"):
            call()


def test_front_end_refuses_gradients():
    x = torch.zeros(1, 1, 1, 64, requires_grad=True)
    pages = torch.zeros(2, 1, 16, 64)
    table, lengths = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: D.cache_write(x, x, pages, pages, table, lengths),
                 lambda: D.tree_attention(x, pages, pages, table, lengths),
                 lambda: D.tree_verify(torch.zeros(1, 2, 5, requires_grad=True), table, None, None, None, greedy=True),
                 lambda: D.quantize_rows(torch.zeros(2, 16, requires_grad=True)),
                 lambda: D.head_logits_int8(x.view(1, 64), torch.zeros(3, 64, dtype=torch.int8), torch.zeros(3))):
        with pytest.raises(RuntimeError, match="gradients are not available"):
            call()


def _m(dtype, shape, dev=0, stride=None):
    """A tensor's metadata as the front end looks at it."""
    if stride is None:
        stride, n = [], 1
        for k in reversed(shape):
            stride.insert(0, n)
            n *= k
    return dtype, dev, torch.Size(shape), tuple(stride)


BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def test_front_end_shapes():
    """What is decided from types, shapes and strides, without a GPU."""
    pages, table, lengths = _m(BF, (9, 2, 16, 64)), _m(I32, (3, 4)), _m(I32, (3,))
    k = _m(BF, (3, 5, 2, 64))
    assert D._write_plan(k, k, pages, pages, table, lengths, None)[1:] == (5, (640, 128, 64), True)
    q = _m(BF, (3, 5, 4, 64))
    c, n, heads, ld, scale, ws = D._attention_plan(q, pages, pages, table, lengths, _m(I32, (3, 5)))
    assert (n, heads, ld, scale, ws) == (5, 4, (1280, 256, 64), 0.125, 0)
    assert (c.pages, c.page_size, c.kv_heads, c.head_dim, c.batch, c.table_pages) == (9, 16, 2, 64, 3, 4)
    wide = _m(I32, (3, 4), stride=(11, 1))
    assert D._attention_plan(q, pages, pages, wide, lengths, None)[0].ld_table == 11
    bad = [
        (k, _m(BF, (3, 4, 2, 64)), pages, pages, table, lengths, None),
        (_m(F32, (3, 5, 2, 64)), k, pages, pages, table, lengths, None),
        (_m(BF, (3, 5, 3, 64)),) * 2 + (pages, pages, table, lengths, None),
        (_m(BF, (2, 5, 2, 64)),) * 2 + (pages, pages, table, lengths, None),
        (_m(BF, (3, 0, 2, 64)),) * 2 + (pages, pages, table, lengths, None),
        (_m(BF, (3, 5, 2, 64), dev=1),) * 2 + (pages, pages, table, lengths, None),
        (_m(BF, (3, 5, 2, 64), stride=(640, 128, 1, 2)),) * 2 + (pages, pages, table, lengths, None),
        (k, k, pages, _m(F32, (9, 2, 16, 64)), table, lengths, None),
        (k, k, pages, _m(BF, (9, 2, 16, 64), stride=(4096, 1024, 64, 1)), table, lengths, None),
        (k, k, _m(BF, (9, 2, 16, 64), stride=(2048, 1024, 1, 16)),
         _m(BF, (9, 2, 16, 64), stride=(2048, 1024, 1, 16)), table, lengths, None),
        (k, k, _m(BF, (1, 9, 2, 16, 64)), _m(BF, (1, 9, 2, 16, 64)), table, lengths, None),
        (k, k, pages, pages, _m(torch.int64, (3, 4)), lengths, None),
        (k, k, pages, pages, _m(I32, (3, 4), stride=(1, 3)), lengths, None),
        (k, k, pages, pages, _m(I32, (3, 4), dev=1), lengths, None),
        (k, k, pages, pages, table, _m(I32, (2,)), None),
        (k, k, pages, pages, table, _m(I32, (3,), stride=(2,)), None),
        (k, k, pages, pages, table, lengths, _m(I32, (4,))),
        (k, k, pages, pages, table, lengths, _m(torch.int64, (3,)))]
    for args in bad:
        with pytest.raises(ValueError):
            D._write_plan(*args)
    with pytest.raises(TypeError):
        D._write_plan(*[_m(torch.float16, (3, 5, 2, 64))] * 2, *[_m(torch.float16, (9, 2, 16, 64))] * 2, table, lengths, None)
    for par in (_m(I32, (3, 4)), _m(torch.int64, (3, 5)), _m(I32, (3, 5), stride=(1, 3))):
        with pytest.raises(ValueError):
            D._attention_plan(q, pages, pages, table, lengths, par)
    for path, acc in ((_m(I32, (3,)), lengths), (_m(I32, (2, 5)), lengths), (_m(I32, (3, 5)), _m(I32, (3, 1)))):
        with pytest.raises(ValueError):
            D._compact_plan(pages, pages, table, lengths, path, acc)
    layers = _m(BF, (7, 9, 2, 16, 64))
    assert D._compact_plan(layers, layers, table, lengths, _m(I32, (3, 5)), lengths)[0].layers == 7


def test_front_end_verification_and_quantization_shapes():
    t, i, u, s = _m(F32, (2, 5, 30)), _m(I32, (2, 5)), _m(F32, (2, 5)), _m(F32, (2,))
    ok = (t, i, i, u, s, t, _m(torch.uint8, (2 * 5 * 20,)), 0.5, 0.75, False)
    assert D._verify_plan(*ok)[:2] == (2, 5)
    for at, x in ((0, _m(BF, (2, 5, 30))), (0, _m(F32, (10, 30))), (0, _m(F32, (2, 5, 30), stride=(150, 31, 1))), (1, None),
                  (1, _m(torch.int64, (2, 5))), (2, _m(I32, (5,))), (3, _m(F32, (5, 2))), (4, _m(F32, (2, 1))),
                  (5, _m(F32, (2, 4, 30))), (6, _m(torch.uint8, (199,))), (6, _m(torch.int8, (200,)))):
        with pytest.raises(ValueError):
            D._verify_plan(*ok[:at], x, *ok[at + 1:])
    assert D._quant_plan(_m(BF, (4, 6), stride=(9, 1))) == (4, 6, 9, B.MLS_BF16)
    for x in (_m(BF, (4,)), _m(BF, (0, 6)), _m(BF, (4, 6), stride=(1, 4)), _m(BF, (4, 6), stride=(0, 1))):
        with pytest.raises(ValueError):
            D._quant_plan(x)
    with pytest.raises(TypeError):
        D._quant_plan(_m(torch.float16, (4, 6)))
    o, W, ws = _m(BF, (3, 32)), _m(torch.int8, (7, 32)), _m(F32, (7,))
    assert D._int8_plan(o, W, ws, None)[:3] == (3, 32, 7)
    for args in ((_m(BF, (3, 16)), W, ws, None), (o, W, _m(F32, (6,)), None), (o, W, ws, _m(F32, (7, 3))),
                 (o, W, ws, _m(BF, (3, 7))), (_m(BF, (3, 32), stride=(33, 1)), W, ws, None)):
        with pytest.raises(ValueError):
            D._int8_plan(*args)
    for args in ((o, _m(torch.uint8, (7, 32)), ws, None), (o, W, _m(BF, (7,)), None)):
        with pytest.raises(TypeError):
            D._int8_plan(*args)


@pytest.mark.parametrize("kw", [
    dict(ld_head=64), dict(ld_head=64 * 15), dict(ld_entry=128), dict(ld_page=1024), dict(ld_page=2048 - 64),
    dict(ld_page=64, ld_head=9 * 64, ld_entry=64), dict(pages=0x7fffffff, ld_page=1 << 48, ld_head=1 << 48)])
def test_entries_that_overlap(kw):
    c = _cache(**kw)
    _refused(B.MLS_INVALID_ARG, _write, c, text="overlap")
    _refused(B.MLS_INVALID_ARG, _compact, c, text="overlap")
    _refused(B.MLS_INVALID_ARG, B.tree_attention_workspace, c, 5, 4, text="overlap")


@pytest.mark.parametrize("kw", [
    dict(ld_head=64, ld_entry=128), dict(ld_page=64, ld_head=9 * 64, ld_entry=18 * 64), dict(ld_entry=72, ld_head=16 * 72, ld_page=32 * 72),
    dict(pages=1, ld_page=0), dict(kv_heads=1, ld_head=0), dict(ld_head=15 * 64 * 2 + 64, ld_entry=128, ld_page=2 * (15 * 128 + 64)),
    dict(pages=0x7fffffff, ld_page=1 << 48)])
def test_dimensions_in_any_order(kw):
    assert B.tree_attention_workspace(_cache(**kw), 5, 4) == 0


def test_strides_of_single_layers_pages_and_heads_do_not_matter():
    table, lengths = _m(I32, (3, 4)), _m(I32, (3,))
    pages = _m(BF, (1, 1, 16, 64), stride=(3, 5, 64, 1))
    k = _m(BF, (3, 5, 1, 64))
    assert D._write_plan(k, k, pages, pages, table, lengths, None)[0].ld_head == 0
    q = _m(BF, (3, 5, 4, 64))
    assert D._attention_plan(q, pages, pages, table, lengths, None)[0].ld_page == 0
    layers = _m(BF, (1, 9, 2, 16, 64), stride=(7, 2048, 1024, 64, 1))
    assert D._compact_plan(layers, layers, table, lengths, _m(I32, (3, 5)), lengths)[0].ld_layer == 0
