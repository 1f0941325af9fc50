"""Limits of the post-training entry points that the host decides. Addresses are made up and never read."""

import pytest

from paper_2608_09703_amd import binding as B

A = 1 << 40


def _problem(T, d=8, V=100):
    return B.make_problem(1, T, V, [d], [A], [2 * A], 3 * A)


def test_tokens_of_one_call():
    """A launch has fewer than 2^32 threads, and a token takes a wave of 64."""
    assert B.token_logp_workspace(_problem((1 << 26) - 128))[0] > 0
    for T in ((1 << 26) - 127, 1 << 26, 1 << 30):
        p = _problem(T)
        for call in (lambda: B.token_logp_workspace(p),
                     lambda: B.token_logp_fwd(p, 4 * A, 5 * A, None, None, 6 * A, 1 << 50, None),
                     lambda: B.token_logp_bwd(p, 4 * A, None, 5 * A, 7 * A, 8 * A, 6 * A, 1 << 50, None)):
            with pytest.raises(B.MlsError, match="2.26") as e:
                call()
            assert e.value.status == B.MLS_UNSUPPORTED


@pytest.mark.parametrize("dtype,n", [(B.MLS_BF16, 8), (B.MLS_F32, 16)])
def test_alignment_of_grad_h(dtype, n):
    p = B.make_problem(1, 100, 500, [64], [A], [2 * A], 3 * A, grad_h_dtype=dtype)
    with pytest.raises(B.MlsError, match="misaligned"):
        B.token_logp_bwd(p, 4 * A, None, 5 * A, 7 * A + n // 2, 8 * A, 6 * A, 1 << 50, None)
