"""Refusals of include/evospec_adapt.h at the ends of what fp32 holds, before anything touches the GPU."""
import pytest

from test_adapt_host import ev, kd, step  # noqa: F401


@pytest.mark.parametrize("eps", [1e-40, 1e-50, 1.17e-38, 5e-324, 3.5e38, 1e300])
def test_eps_that_fp32_does_not_have(ev, eps):  # noqa: F811
    """Its reciprocal would be infinite: elements that never had a gradient became 0 x infinity."""
    assert step(ev, eps=eps) == 2


def test_the_least_and_the_largest_eps(ev):  # noqa: F811
    nothing = ((None, None, 0),)
    assert step(ev, rows=nothing, eps=2.0 ** -126) == 0 and step(ev, rows=nothing, eps=3e38) == 0


@pytest.mark.parametrize("T", [1e-39, 1e-45, 1.17e-38])
def test_temperatures_whose_reciprocal_is_infinite(ev, T):  # noqa: F811
    assert kd(ev, T=T) == 2 and kd(ev, T=2.0 ** -126, E=0) == 0 and kd(ev, T=3e38, E=0) == 0


def test_moments_of_more_than_one_launch(ev):  # noqa: F811
    """As many blocks as several of the largest tensors have are no bad size: the call goes on to what it is given."""
    f = ev.lib.evospec_adamw_moments
    assert f(16, 16, 8, (1 << 25) + 1, 0, None, 16, None) == 1 and f(16, 16, 8, 1 << 30, 0, 16, 8, None) == 4 and f(16, 16, 8, (1 << 40) + 1, 0, 16, 16, None) == 2
