"""CPU: the values of a step's rule that are refused.  Whatever is in order reaches the missing context."""
import pytest

from test_list_host import INVALID, lib, param, rule, step  # noqa: F401

SHAPE = -2


def taken(lib, **kw):  # noqa: F811
    # (a rule is looked at before the arrays: one with a negative size answers for a rule that is in order)
    got = step(lib, param(rows=-1), r=rule(**kw))
    assert got in (INVALID, SHAPE)
    return got == SHAPE


@pytest.mark.parametrize("eps", [0.0, 1e-8, 1e-30, 2.0 ** -126, 1.0, 2.0 ** 125])
def test_eps_that_is_taken(lib, eps):  # noqa: F811
    assert taken(lib, eps=eps)


@pytest.mark.parametrize("eps", [5e-324, 1e-50, 1e-45, 1e-40, 2.0 ** -126 * (1 - 2.0 ** -50), 2.0 ** 125 * (1 + 2.0 ** -50), 2.0 ** 126, 1e39, 1e300,
                                 float("inf"), -float("inf"), float("nan"), -1e-8, -1e-300])
def test_eps_that_is_refused(lib, eps):  # noqa: F811
    # fp32 holds it with fewer bits or not at all, or the quotient's bound does not reach so far
    assert not taken(lib, eps=eps)
    assert step(lib, param(rows=-1), r=rule(eps=eps), adamw=False) == SHAPE      # Lion has none
