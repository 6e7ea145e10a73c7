"""Gated projections on rows as far apart as the library allows, and their backward against the linear layer's with [dg du] made outside."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from tests import dispatch_host
from tests.test_gpu_gated import HALF, U, _draw, _f64, _within
from tests.test_gpu_gated_tiles import FEW, MIDDLE, RULES, SHORT

PITCH = 1 << 22
SHAPES = {FEW: (32, 128, 64), SHORT: (65, 128, 64), MIDDLE: (200, 128, 8256)}


def test_shapes_take_the_kernels():
    assert [r[0] for r in dispatch_host.ask(SHAPES.values(), *RULES, names=("M", "K", "F"))] == list(SHAPES)


def _far(t):
    """A copy of the matrix whose rows are PITCH elements apart."""
    rows, cols = t.shape
    out = torch.empty((rows - 1) * PITCH + cols, dtype=t.dtype, device="cuda").as_strided((rows, cols), (PITCH, 1))
    return out.copy_(t)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,F", SHAPES.values())
def test_rows_far_apart(M, K, F):
    """Offsets of up to 2^22 elements a row: the bits of the call on contiguous rows."""
    from paper_2507_00394_amd import binding as hx

    a, w, dh = _draw(1, (M, K)), _draw(2, (K, 2 * F), K ** -0.5), _draw(3, (M, F))
    ws = torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F), dtype=torch.uint8, device="cuda")
    results = []
    for place in (lambda t: t, _far):
        nan = lambda *s: place(torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda"))
        x, y, z, h, gu = place(a), place(w), place(dh), nan(M, F), nan(M, 2 * F)
        hx.helix_gated_linear_fwd(x, y, h, gu=gu)
        out = [h, gu]
        for kept in (None, gu):
            da, dw = nan(M, K), nan(K, 2 * F)
            hx.helix_gated_linear_bwd(x, y, z, da, dw, ws, gu=kept)
            out += [da, dw]
        results.append([t.contiguous() for t in out])
        del x, y, z, h, gu, da, dw, out
    assert all(torch.equal(p, q) and torch.isfinite(p).all() for p, q in zip(*results))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", [(32, 256, 128), (320, 256, 192), (1504, 640, 704)])
def test_backward_is_the_linear_layers_of_dgu(M, K, F, kind):
    """[dg du] of the kept projections, made in 64 bits and rounded to bf16, through helix_qkv_linear_bwd.  The gated call's own [dg du] are of fp32 arithmetic: where they lie next to the middle between two
    bf16 numbers they can be the other of the two, 2 * HALF of the value away."""
    from paper_2507_00394_amd import binding as hx

    a, w, dh = _draw(1, (M, K)), _draw(2, (K, 2 * F), 1.5 * K ** -0.5), _draw(3, (M, F))
    gu, h, da, dw = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((M, 2 * F), (M, F), (M, K), (K, 2 * F)))
    hx.helix_gated_linear_fwd(a, w, h, gu=gu, activation=kind)
    hx.helix_gated_linear_bwd(a, w, dh, da, dw, torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F), dtype=torch.uint8, device="cuda"), gu=gu, activation=kind)
    dgu = torch.from_numpy(R.gated_bwd_ref(_f64(a), _f64(w), _f64(dh), kind, _f64(gu))[2]).to(torch.bfloat16).cuda()
    da2, dw2 = torch.empty_like(da), torch.empty(K, 2 * F, device="cuda")
    hx.helix_qkv_linear_bwd(a, w, dgu, da2, dw2, torch.empty(hx.helix_qkv_linear_bwd_workspace_bytes(M, K, 2 * F), dtype=torch.uint8, device="cuda"))
    size = np.abs(_f64(dgu))
    for name, got, ref, total, terms in (("da", da, da2, size @ np.abs(_f64(w)).T, 2 * F), ("dw", dw, dw2, np.abs(_f64(a)).T @ size, M)):
        ref = _f64(ref)
        off = (2 * HALF + 2 * (terms + 40) * U) * total
        _within(name, got, ref, 2 * HALF * (np.abs(ref) + off) + off, norm=True)
