"""The gated projections' activation and its derivative, point by point, in the negative tail too, in every kernel that evaluates them.

One column of either half of w has a one, so that g is an element of a and u is 1: h is act(g), and with dh = 1 the first two columns of da are act'(g) and act(g), each rounded once.
Tolerance: HALF = 2^-8 of the value for its rounding to bf16.  In fp32 the exponential's argument, at most 72 here (12^2 / 2), has three roundings, 72 * 3 * 2^-24 = 1.3e-5 of the value; the polynomial's
1.5e-7 and about twenty roundings more make 1.5e-5, below 2^-16: 2^-15 of the value is allowed.  The derivative has a zero between -2 and 0, where terms of the size of 1 cancel: 16 roundings of 2^-24 there."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from tests import dispatch_host
from tests.test_gpu_gated_tiles import FEW, MIDDLE, RULES, SHORT, WIDE

HALF = 2.0 ** -8
SHAPES = {FEW: (32, 128, 64), SHORT: (700, 128, 64), MIDDLE: (700, 128, 8192), WIDE: (5000, 256, 1408)}


def test_shapes_take_every_kernel():
    assert [r[0] for r in dispatch_host.ask(SHAPES.values(), *RULES, names=("M", "K", "F"))] == list(SHAPES)


def _points(M):
    """bf16 values from -12 to 12, exact zero among them."""
    g = torch.linspace(-12, 12, M, dtype=torch.float64)
    g[M // 2] = 0
    return g.to(torch.bfloat16).cuda()


def _check(name, got, ref, g):
    got, off = got.double().cpu().numpy(), 2.0 ** -15 * np.abs(ref) + (np.abs(g) < 2) * 16 * 2.0 ** -24
    over = np.abs(got - ref) - (HALF * (np.abs(ref) + off) + off)
    at = over.argmax()
    assert over[at] <= 0, f"{name}({g[at]}) = {got[at]}, {ref[at]} in 64 bits"


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", SHAPES.values())
def test_values_and_slopes(M, K, F, kind):
    from paper_2507_00394_amd import binding as hx

    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    for column in (0, F - 1):
        a, w = torch.zeros(M, K, **bf16), torch.zeros(K, 2 * F, **bf16)
        a[:, 0], a[:, 1] = _points(M), 1
        w[0, column] = w[1, F + column] = 1
        g = a[:, 0].double().cpu().numpy()
        value, slope = R.activation_ref(g, kind)
        gu, h, da, dw = (torch.empty(s, **bf16) for s in ((M, 2 * F), (M, F), (M, K), (K, 2 * F)))
        hx.helix_gated_linear_fwd(a, w, h, gu=gu, activation=kind)
        assert torch.equal(gu[:, column], a[:, 0]) and (gu[:, F + column] == 1).all()
        _check("act", h[:, column], value, g)
        ws = torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F), dtype=torch.uint8, device="cuda")
        for kept in (None, gu):
            hx.helix_gated_linear_bwd(a, w, torch.ones(M, F, **bf16), da, dw, ws, gu=kept, activation=kind)
            _check("slope", da[:, 0], slope, g)
            _check("act in the backward", da[:, 1], value, g)
