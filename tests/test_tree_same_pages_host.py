"""Keys and values written to the same pages are refused; the same entries, or pages that are read alone, are not."""

from paper_2608_09703_amd import binding as B
from tests.test_tree_abi_host import _at, _cache, _refused, _write


def test_keys_and_values_in_the_same_pages():
    c = _cache(v=_at(1))
    _refused(B.MLS_INVALID_ARG, _write, c, text="same pages")
    assert B.tree_attention_workspace(c, 5, 4) == 0
    # (what stops this one is its first address)
    _refused(B.MLS_INVALID_ARG, lambda: _write(c, k=_at(5, 8), v=_at(5, 8)), text="aligned")
