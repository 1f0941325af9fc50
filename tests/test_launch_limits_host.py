"""Calls of more threads than one launch takes (2^32 along a dimension of the grid; it runs a part of them and reports
nothing) are refused on the host. Addresses are made up and never read."""

import pytest

from paper_2608_09703_amd import binding as B
from tests.test_tree_abi_host import _at, _refused


@pytest.mark.parametrize("prev,fresh,T", [(8, 1024, 1 << 26), (1032, 8, 1 << 25), (2056, 2048, 1 << 24), (8192, 8, 1 << 24)])
def test_junction(prev, fresh, T):
    j = lambda T: B.make_junction(T, prev, fresh)  # noqa: E731
    _refused(B.MLS_UNSUPPORTED, B.junction_fwd, j(T), _at(1), _at(2), _at(3), None, text="one launch")
    _refused(B.MLS_UNSUPPORTED, B.junction_bwd, j(T), _at(1), _at(2), _at(3), _at(4), _at(5), None, text="one launch")
    # (what stops the next smaller one is its misaligned address)
    _refused(B.MLS_INVALID_ARG, B.junction_fwd, j(T - 1), _at(1, 8), _at(2), _at(3), None, text="aligned")


def test_chain_verification():
    s, g = B.make_sampling(4), B.make_sampling(4, greedy=True)
    call = lambda s, batch, gamma, rec=None: B.spec_verify(  # noqa: E731
        s, batch, gamma, _at(1), _at(2), _at(3), _at(4), _at(5), _at(6), _at(7), _at(8), 1 << 33, None, draft_params=rec)
    _refused(B.MLS_INVALID_ARG, B.spec_verify_workspace, 1 << 22, 0)
    _refused(B.MLS_INVALID_ARG, call, g, 1 << 22, 0)
    _refused(B.MLS_UNSUPPORTED, call, s, (1 << 22) // 7 + 1, 3, text="2^22")
    _refused(B.MLS_UNSUPPORTED, call, s, 1 << 20, 3, _at(9), text="2^22")


def test_head():
    _refused(B.MLS_UNSUPPORTED, B.head_logits, 1, 1 << 30, 8, B.MLS_BF16, _at(1), _at(2), _at(3), None, text="one launch")
    _refused(B.MLS_UNSUPPORTED, B.head_logits, 1 << 25, 128 * 64, 8, B.MLS_F32, _at(1), _at(2), _at(3), None, text="one launch")
