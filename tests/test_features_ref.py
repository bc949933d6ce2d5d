"""The comparison that the operators on point features are tested with rejects what it has to."""
import pytest
import torch

from tests import features_ref as F

INF, NAN = float("inf"), float("nan")


def _want():
    ref = torch.tensor([[1.0, -2.0, 0.0], [4.0, 5.0, -6.0]], dtype=torch.float64)
    return ref, torch.full((2, 1), 0.25, dtype=torch.float64)


def _put(x, value, at=(1, 1)):
    x = x.clone()
    x[at] = value
    return x


def test_check_takes_what_is_within_the_bounds():
    ref, bound = _want()
    F.check({"x": ref}, {"x": (ref, bound)}, "same")
    F.check({"x": ref + 0.25}, {"x": (ref, bound)}, "at the bound")
    F.check({"x": ref.float()}, {"x": (ref, bound)}, "of another type")
    for odd in (INF, -INF, NAN):
        F.check({"x": _put(ref, odd)}, {"x": (_put(ref, odd), bound)}, "not finite alike")
    F.check({"x": torch.zeros(0, 3)}, {"x": (torch.zeros(0, 3, dtype=torch.float64), torch.zeros(0, 1))}, "nothing")


@pytest.mark.parametrize("value", [NAN, INF, -INF, 5.2501, 4.7499])
def test_check_rejects_a_value(value):
    ref, bound = _want()
    with pytest.raises(AssertionError):
        F.check({"x": _put(ref, value)}, {"x": (ref, bound)}, "one")
    with pytest.raises(AssertionError):
        F.check({"x": torch.full_like(ref, value)}, {"x": (ref, bound)}, "all")


@pytest.mark.parametrize("odd", [INF, -INF, NAN])
@pytest.mark.parametrize("value", [0.0, INF, -INF, NAN])
def test_check_rejects_another_value_than_one_that_is_not_finite(odd, value):
    ref, bound = _want()
    if value == odd or value != value and odd != odd:
        return
    with pytest.raises(AssertionError):
        F.check({"x": _put(ref, value)}, {"x": (_put(ref, odd), bound)}, "odd")


@pytest.mark.parametrize("value", [NAN, INF])
def test_check_rejects_a_bound_that_is_not_finite(value):
    ref, bound = _want()
    with pytest.raises(AssertionError):
        F.check({"x": ref}, {"x": (ref, torch.full_like(bound, value))}, "bound")


def test_check_rejects_a_shape_or_a_name():
    ref, bound = _want()
    with pytest.raises(AssertionError):
        F.check({"x": ref[:1]}, {"x": (ref, bound)}, "shape")
    with pytest.raises(KeyError):
        F.check({"y": ref}, {"x": (ref, bound)}, "name")
