"""Gated projections whose input gradient has so long a contraction that it is cut into parts, and the largest and smallest widths."""
import pytest

from tests import dispatch_host
from tests.test_gpu_gated import _check_backward, _check_forward

SHAPES = [(1, 128, 3200), (33, 256, 3136), (70, 128, 3264), (300, 384, 4096), (4096, 128, 3200)]


def test_the_contraction_is_in_parts():
    assert all(p > 1 for p, in dispatch_host.ask([(m, k, 2 * f) for m, k, f in SHAPES], "split_input_parts(M, K, N)", names=("M", "K", "N")))
    assert dispatch_host.ask([(4097, 128, 6400), (300, 384, 6016)], "split_input_parts(M, K, N)", names=("M", "K", "N")) == [(1,), (1,)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,F", SHAPES)
def test_long(M, K, F):
    a, w, gu = _check_forward(M, K, F, "silu", pads=(16, 2))
    _check_backward(M, K, F, "silu", a, w, gu, pads=(16, 2))
