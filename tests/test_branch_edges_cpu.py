"""Calls for branches of one context where they can go wrong, without a GPU."""
import pytest

from test_branches_cpu import CTX, SHAPE, lib, rope  # noqa: F401


@pytest.mark.parametrize("want,eps", [(CTX, 1.2e-38), (CTX, 1e-6), (SHAPE, 1.1e-38), (SHAPE, 1e-45), (SHAPE, -1e-6)])
def test_rope_refuses_an_eps_that_the_norm_takes_for_zero(lib, want, eps):  # noqa: F811
    assert rope(lib, eps=eps) == want, lib.sa_last_error()
