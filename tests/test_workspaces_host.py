"""Workspace sizes of the operators around the attention stage (no GPU): enough for what a call of as many rows or fewer writes, and no more than the largest of those."""
import numpy as np
import pytest

from paper_2507_00394_amd import binding as hx
from tests import dispatch_host as H


@pytest.fixture(scope="module", autouse=True)
def library():
    if not hx.LIB_PATH.exists():
        from paper_2507_00394_amd import build

        build.build()
    return hx.lib()


def _up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("E", [1, 64, 256, 257, 1000, 1024, 1025, 2048, 4096, 5000, 16384])
def test_layer_norm(E):
    rows = [*range(1, 5000), 16384, 131072, 2 ** 31 - 1]
    sizes = [hx.helix_layer_norm_bwd_workspace_bytes(M, E) for M in rows]
    slabs = [n for n, in H.ask([(M, E) for M in rows], "norm_bwd_groups(rows, cols)", names=("rows", "cols"))]
    assert sizes == [_up(int(n) * 2 * 4 * E) for n in np.maximum.accumulate(slabs)]
    assert max(sizes) == _up(256 * 2 * 4 * E)


@pytest.mark.parametrize("K,F", [(128, 64), (128, 3200), (512, 3840), (2048, 5504), (5120, 3136), (4096, 11008), (5120, 1728), (1024, 3136)])
def test_gated_projections(K, F):
    rows = [*range(1, 4500), *range(4501, 140000, 997)]
    sizes = [hx.helix_gated_linear_bwd_workspace_bytes(M, K, F) for M in rows]
    parts = H.ask([(M, K, 2 * F) for M in rows], "split_weight_parts(M, K, N)", "split_input_parts(M, K, N)", names=("M", "K", "N"))
    slabs = np.maximum.accumulate([max(q * K * 2 * F * 4 if q > 1 else 0, p * M * K * 4 if p > 1 else 0) for M, (q, p) in zip(rows, parts)])
    transposed = _up(K * 2 * F * 2)
    assert sizes == [_up(_up(transposed + int(s)) + -(-M // 32) * 32 * 2 * F * 2) for M, s in zip(rows, slabs)]
