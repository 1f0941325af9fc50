"""Sizes past what one launch takes (2^32 threads along a dimension of the grid) are refused on the host, before any
kernel runs; addresses are made up and never read."""

import pytest

from paper_2608_09703_amd import binding as B
from tests.test_tree_abi_host import _at, _attend, _cache, _refused, _verify, _write


def test_trees():
    s = B.make_sampling(2, greedy=True)
    assert B.tree_verify_workspace(s, (1 << 22) - 1, 1) == 0
    _refused(B.MLS_INVALID_ARG, B.tree_verify_workspace, s, 1 << 22, 1)
    _refused(B.MLS_INVALID_ARG, lambda: _verify(V=2, batch=1 << 22, n=1, greedy=True))


@pytest.mark.parametrize("kw,n,heads,more", [
    # 65 parts each: 7 x 65 x 32,768 blocks, a multiple of 8; the eighth head passes 2^24
    (dict(batch=32768, kv_heads=7, table_pages=16400, ld_table=16400), 1, 7, dict(kv_heads=8)),
    (dict(batch=65535, kv_heads=256), 1, 256, dict(kv_heads=257)),  # one part each
    # 1,024 rows a key head: 8 blocks of 128
    (dict(batch=32767, kv_heads=64, table_pages=64, ld_table=64), 64, 1024, dict(batch=32768))])
def test_blocks_of_attention(kw, n, heads, more):
    B.tree_attention_workspace(_cache(**kw), n, heads)
    c = _cache(**dict(kw, **more))
    heads = heads // kw["kv_heads"] * c.kv_heads
    _refused(B.MLS_UNSUPPORTED, B.tree_attention_workspace, c, n, heads, text="one launch")
    _refused(B.MLS_UNSUPPORTED, lambda: _attend(c, n=n, heads=heads), text="one launch")


def test_rows_to_join():
    # 65,535 x 1 x 4,096 x 64 / 4 threads are 2^32 less 65,536; with heads of 96 they are more
    kw = dict(kv_heads=1, table_pages=512, ld_table=512, page_size=16)
    c = _cache(batch=65535, head_dim=64, **kw)
    assert B.tree_attention_workspace(c, 1, 4096) > 0
    _refused(B.MLS_UNSUPPORTED, B.tree_attention_workspace, _cache(batch=65535, head_dim=96, **kw), 1, 4096, text="joins")
    one = dict(kw, table_pages=16, ld_table=16)  # nothing to join
    B.tree_attention_workspace(_cache(batch=65535, head_dim=96, **one), 1, 4096)


def test_entries_written():
    c = _cache(kv_heads=65536, head_dim=8, ld_head=128, ld_page=65536 * 128, ld_entry=8)
    # (n / 16 + 1) 8,192 blocks: n = 32,736 makes 2,047 of them
    _refused(B.MLS_INVALID_ARG, lambda: _write(c, n=32752, ld=(0, 0, 8)), text="out of range")
    _refused(B.MLS_INVALID_ARG, lambda: _write(_cache(), n=1 << 28), text="out of range")


def test_tiles_of_the_8_bit_head():
    h = lambda T, V: B.head_logits_int8(T, V, 32, B.MLS_BF16, _at(1), _at(2), _at(3), _at(4), _at(5), 1 << 40, None)  # noqa: E731
    _refused(B.MLS_INVALID_ARG, h, 1, 1 << 30, text="out of range")  # tiles of 64 x 32
    _refused(B.MLS_INVALID_ARG, h, 1 << 25, 192 * 64, text="out of range")  # of 192 x 128
