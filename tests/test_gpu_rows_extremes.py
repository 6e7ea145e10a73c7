"""Layer norm on rows whose mean is so large that mean * rstd has no fp32 value, though every element's (x - mean) * rstd has."""
import pytest
import torch

from tests.test_gpu_rows import TYPES, _draw, _params

pytestmark = pytest.mark.gpu


# columns behind the last whole chunk alone, with a chunk, lanes without a chunk, both, and two chunks a lane at most
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("E", [5, 9, 64, 100, 128])
def test_constant_rows_of_large_values(kind, E):
    """x = 2^120 throughout: xh = 0, so dx = rstd * (g - mean(g)), dgamma = 0 and dbeta the sum of dy.  64 roundings of 2^-24 for the mean of |g| and the rest."""
    from paper_2507_00394_amd import binding as hx

    M, dtype = 40, TYPES[kind]
    x, dy, (gamma, beta) = torch.full((M, E), 2.0 ** 120, dtype=dtype, device="cuda"), _draw(E, M, E, dtype), _params(E)
    mean, rstd = torch.full((M,), 2.0 ** 120, device="cuda"), torch.full((M,), 1e-5 ** -0.5, device="cuda")
    assert torch.isinf(mean * rstd).all()
    ws = torch.empty(hx.helix_layer_norm_bwd_workspace_bytes(M, E), dtype=torch.uint8, device="cuda")
    g = dy.double() * gamma.double()
    want = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    off = 64 * 2.0 ** -24 * rstd.double()[:, None] * (g.abs() + g.abs().mean(1, keepdim=True))
    tol = torch.finfo(dtype).eps / 2 * (want.abs() + off) + off
    for both in (False, True):
        dx, dr = torch.empty_like(x), torch.empty_like(x)
        dgamma, dbeta = (torch.full((E,), float("nan"), device="cuda") for _ in range(2))
        if both:
            hx.helix_dropout_add_layer_norm_bwd(dy, None, x, gamma, mean, rstd, dx, dr, dgamma, dbeta, ws, 0.0, None)
            assert torch.equal(dx, dr)
        else:
            hx.helix_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
        assert ((dx.double() - want).abs() <= tol).all()
        assert (dgamma == 0).all() and ((dbeta.double() - dy.double().sum(0)).abs() <= M * 2.0 ** -24 * dy.double().abs().sum(0)).all()
