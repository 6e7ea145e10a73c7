"""Gated projections on every tile of the forward and every pair of gradient kernels that the rules can pick, the 256 x 128 tile of training sizes among them.  The tests without a GPU ask the
rules (csrc/dispatch.hpp) which kernels the shapes select, so that a change of a rule cannot take a kernel out of the tests unseen."""
import pytest

from tests import dispatch_host
from tests.test_gpu_gated import _check_backward, _check_forward

FEW, WIDE, MIDDLE, SHORT = -1, 0, 1, 2     # at most 32 rows; tiles of 256 x 128, 128 x 64 and 64 x 64 elements of h
RULES = ("gated_few(M, F) ? -1 : (int)gated_tile(M, K, F)",
         "split_input_parts(M, K, 2 * F) > 1 ? 3 + (int)split_input_tile(M) : (int)linear_gradient_tiles(M, K, 2 * F, split_weight_parts(M, K, 2 * F)).input",
         "(int)linear_gradient_tiles(M, K, 2 * F, split_weight_parts(M, K, 2 * F)).weight", "split_weight_parts(M, K, 2 * F) > 1")

# 256 x 128 tiles: whole in both directions; cut in M, in F, in both; one row in the last row of tiles
WIDE_SHAPES = [(4096, 256, 1792), (5000, 256, 1408), (4096, 256, 1728), (5003, 384, 1472), (4097, 256, 1728)]

# input gradient (256, 128 and 64 tiles, or in parts on 128 and 64 tiles), weight gradient (256, 128, 64), whether it is in parts
PAIR_SHAPES = {(0, 0, 0): (1500, 5120, 704), (0, 0, 1): (20001, 256, 1088), (1, 0, 0): (300, 5120, 1408), (1, 0, 1): (7001, 384, 2944), (1, 1, 0): (201, 5120, 192),
               (1, 1, 1): (4100, 2048, 128), (1, 2, 0): (513, 128, 64), (1, 2, 1): (4100, 128, 64), (2, 0, 0): (5, 5120, 2752), (2, 1, 0): (9, 128, 320), (2, 1, 1): (4100, 128, 1728),
               (2, 2, 0): (1, 128, 64), (2, 2, 1): (4100, 128, 576), (4, 0, 0): (100, 5120, 3136), (4, 0, 1): (4096, 512, 3840), (4, 1, 0): (67, 128, 3136), (4, 1, 1): (4096, 128, 3136),
               (5, 0, 0): (5, 4096, 3136), (5, 1, 0): (1, 128, 3136)}


def _ask(shapes):
    return dispatch_host.ask(shapes, *RULES, names=("M", "K", "F"))


def test_wide_shapes_take_the_wide_tile():
    assert [r[0] for r in _ask(WIDE_SHAPES)] == [WIDE] * len(WIDE_SHAPES)
    assert {(bool(M % 256), bool(F % 128)) for M, _, F in WIDE_SHAPES} == {(a, b) for a in (False, True) for b in (False, True)}


def test_each_pair_is_the_one_named():
    assert [r[1:] for r in _ask(PAIR_SHAPES.values())] == list(PAIR_SHAPES)
    assert all(M % 32 for (_, _, parts), (M, _, _) in PAIR_SHAPES.items() if M != 4096)     # 4096: the only length with both products in parts


def test_no_tile_and_no_pair_is_left_out():
    rows = (1, 5, 16, 31, 32, 33, 64, 65, 100, 128, 200, 257, 300, 513, 700, 1000, 1500, 2049, 3000, 4096, 4097, 5000, 7001, 10001, 20001, 32768, 65537, 131072)
    found = _ask([(M, 128 * k, 64 * f) for M in rows for k in (1, 2, 3, 4, 6, 8, 12, 16, 20, 23, 25, 32, 40) for f in (1, 2, 3, 5, 9, 11, 17, 22, 27, 33, 43, 46, 49, 60, 63, 86, 128, 129, 172)])
    assert {r[0] for r in found} == {r[0] for r in _ask([*WIDE_SHAPES, *PAIR_SHAPES.values()])} == {FEW, WIDE, MIDDLE, SHORT}
    assert {r[1:] for r in found} == set(PAIR_SHAPES)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", WIDE_SHAPES)
def test_wide_tile(M, K, F, kind):
    a, w, gu = _check_forward(M, K, F, kind, pads=(16, 3))
    _check_backward(M, K, F, kind, a, w, gu, pads=(32, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,F", PAIR_SHAPES.values())
def test_pair(M, K, F):
    a, w, gu = _check_forward(M, K, F, "silu", pads=(16, 2))
    _check_backward(M, K, F, "silu", a, w, gu, pads=(16, 2))
