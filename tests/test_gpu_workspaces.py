"""The backward calls of the operators around the attention stage write nothing around a workspace of the size that they name, and every output of theirs, in place too."""
import pytest
import torch

from tests.test_gpu_gated import _draw as _bf16
from tests.test_gpu_gated_tiles import PAIR_SHAPES, WIDE_SHAPES
from tests.test_gpu_rows import TYPES, _draw, _params, _rng

pytestmark = pytest.mark.gpu
GUARD, MARK = 1 << 16, 0xA5


def _guarded(n):
    """(buffer, the n bytes in the middle of it), filled with a mark."""
    buf = torch.full((n + 2 * GUARD,), MARK, dtype=torch.uint8, device="cuda")
    return buf, buf[GUARD:GUARD + n]


def _untouched(buf):
    assert (buf[:GUARD] == MARK).all() and (buf[-GUARD:] == MARK).all()


# a single workgroup; one wave's rows to each of up to 256 workgroups; more rows to a workgroup; all of them
@pytest.mark.parametrize("M,E", [(1, 16384), (17, 2048), (128, 256), (129, 256), (256, 1111), (257, 1111), (513, 5000), (1024, 200), (1025, 200), (3001, 1024), (5000, 4096), (700, 16384)])
def test_around_the_norms_workspace(M, E):
    from paper_2507_00394_amd import binding as hx

    x, dy, (gamma, beta) = _draw(1, M, E, torch.bfloat16), _draw(2, M, E, torch.bfloat16), _params(E)
    y, dx, dr = (torch.empty_like(x) for _ in range(3))
    mean, rstd, dgamma, dbeta = (torch.empty(n, device="cuda") for n in (M, M, E, E))
    hx.helix_layer_norm_fwd(x, gamma, beta, y, mean, rstd)
    buf, ws = _guarded(hx.helix_layer_norm_bwd_workspace_bytes(M, E))
    hx.helix_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    _untouched(buf)
    hx.helix_dropout_add_layer_norm_bwd(dy, None, x, gamma, mean, rstd, dx, dr, dgamma, dbeta, ws, 0.1, _rng())
    _untouched(buf)


@pytest.mark.parametrize("M,K,F", [*PAIR_SHAPES.values(), WIDE_SHAPES[3], (32, 128, 64), (33, 4096, 8192)])
def test_around_the_projections_workspace(M, K, F):
    from paper_2507_00394_amd import binding as hx

    a, w, dh = _bf16(1, (M, K)), _bf16(2, (K, 2 * F), 0.05), _bf16(3, (M, F))
    gu, h, da, dw = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((M, 2 * F), (M, F), (M, K), (K, 2 * F)))
    hx.helix_gated_linear_fwd(a, w, h, gu=gu)
    buf, ws = _guarded(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F))
    for kept in (gu, None):
        hx.helix_gated_linear_bwd(a, w, dh, da, dw, ws, gu=kept)
        _untouched(buf)


def test_the_largest_batchs_workspace_does_for_the_others():
    from paper_2507_00394_amd import binding as hx

    E, (K, F), most = 2048, (128, 3200), 4200
    ws = torch.empty(max(hx.helix_layer_norm_bwd_workspace_bytes(most, E), hx.helix_gated_linear_bwd_workspace_bytes(most, K, F)), dtype=torch.uint8, device="cuda")
    gamma, w = torch.ones(E, device="cuda"), _bf16(1, (K, 2 * F), 0.05)
    for M in (most, 4096, 2000, 256, 65, 64, 1):
        x, a, dh = _draw(M, M, E, torch.bfloat16), _bf16(M, (M, K)), _bf16(M + 1, (M, F))
        stat = lambda n: torch.zeros(n, device="cuda")
        norm = lambda ws: hx.helix_layer_norm_bwd(x, x, gamma, stat(M), stat(M) + 1, out[0], out[1], out[2], ws)
        gated = lambda ws: hx.helix_gated_linear_bwd(a, w, dh, out[3], out[4], ws)
        results = []
        for own in (True, False):
            out = [torch.empty_like(x), stat(E), stat(E), torch.empty_like(a), torch.empty_like(w)]
            new = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
            norm(new(hx.helix_layer_norm_bwd_workspace_bytes(M, E)) if own else ws)
            gated(new(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F)) if own else ws)
            results.append(out)
        assert all(torch.equal(p, q) for p, q in zip(*results)), M


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,E", [(3, 7), (40, 520), (300, 5001)])
def test_in_place_calls_write_the_statistics_and_the_parameters_gradients(kind, M, E):
    """All of them were NaN before the call, and are the bits of the call that is not in place."""
    from paper_2507_00394_amd import binding as hx

    dtype, rng, (gamma, beta) = TYPES[kind], _rng(), _params(E)
    src = [_draw(n, M, E, dtype) for n in range(3)]
    new = lambda n: torch.full((n,), float("nan"), device="cuda")
    ws = torch.full((hx.helix_layer_norm_bwd_workspace_bytes(M, E),), 255, dtype=torch.uint8, device="cuda")
    mean, rstd = new(M), new(M)
    hx.helix_layer_norm_fwd(src[1], gamma, beta, torch.empty_like(src[1]), mean, rstd)

    def norm(i, o, f):
        hx.helix_layer_norm_fwd(i[1], gamma, beta, o[0], *f)

    def norm_bwd(i, o, f):
        hx.helix_layer_norm_bwd(i[0], i[1], gamma, mean, rstd, o[0], *f, ws)

    def both(i, o, f):
        hx.helix_dropout_add_layer_norm_fwd(i[0], i[1], o[0], gamma, beta, o[1], *f, 0.3, rng)

    def both_bwd(i, o, f):
        hx.helix_dropout_add_layer_norm_bwd(i[0], i[2], i[1], gamma, mean, rstd, o[0], o[1], *f, ws, 0.3, rng)

    for call, length, places in ((norm, M, [(1,)]), (norm_bwd, E, [(0,), (1,)]), (both, M, [(1, 0), (0, 1)]), (both_bwd, E, [(0, 2), (2, 0), (1, 2)])):
        want = new(length), new(length)
        call(src, [torch.empty_like(src[0]) for _ in range(2)], want)
        assert all(torch.isfinite(t).all() for t in want)
        for place in places:     # the inputs whose places the outputs take
            inputs, got = [t.clone() for t in src], (new(length), new(length))
            call(inputs, [inputs[p] for p in place], got)
            assert all(torch.equal(a, b) for a, b in zip(want, got)), (call.__name__, place)
