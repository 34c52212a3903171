"""Refusals of libdscores at the ends of its ranges, on the host."""
import pytest

sc = pytest.importorskip("paper_1111_1373_amd.scores", reason="libdscores.so not built")

from tests.test_scores_cpu import INVALID, _backward, _distill  # noqa: E402


@pytest.mark.parametrize("t", [2.0 ** 60 * (1 + 2.0 ** -23), 1e20, 3.4e38, 4.4e-39, 0.0])
def test_temperatures_out_of_range(t):
    assert _distill(t=t) == INVALID
    assert _backward(t=t) == INVALID
    assert b"temperature" in sc._lib.ds_last_error()


@pytest.mark.parametrize("t", [2.0 ** 60, 1.0, 1e-38, 4.5e-39])
def test_temperatures_in_range(t):
    none = dict(x=None, n=0, values=None, index=None, g=None, stats=None, grad=None)
    assert _distill(**none, loss=None, t=t) == 0
    assert _backward(**none, t=t) == 0
