"""Gated projections on the GPU against the fp64 oracle.

Tolerances.  A sum of n products in fp32 is off by at most n * 2^-24 of the sum of their magnitudes; bf16 rounds by at most HALF = 2^-8 relative to
the value.  h = act(g) u is then off by |act'| |u| off(g) + |act| off(u), a few fp32 roundings (16 * 2^-24 of |h|, |g u| for what cancels
inside the activation) and its own rounding; |act'| <= 1.13.  da and dw are sums of products with dg and du, which are rounded to bf16: HALF of
the sum of magnitudes, and their own rounding.  Over a whole matrix these two roundings are independent: the 2-norm of the error is below
2 * HALF / sqrt(3) = 1.2 HALF of that of the result if every rounding were of a value just above a power of two, and about half of that in fact: HALF is allowed."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from paper_2507_00394_amd import inputs as I

pytestmark = pytest.mark.gpu
HALF, U = 2.0 ** -8, 2.0 ** -24
NAN = float("nan")


def _draw(seed, shape, std=1.0):
    g = np.random.Generator(np.random.Philox(seed))
    return torch.from_numpy(g.standard_normal(shape) * std).to(torch.bfloat16).cuda()


def _f64(t):
    return t.detach().double().cpu().numpy()


def _nan(rows, cols, pad_cols=0, pad_rows=0):
    buf = torch.full((rows + pad_rows, cols + pad_cols), NAN, dtype=torch.bfloat16, device="cuda")
    return buf, buf[:rows, pad_cols // 2:pad_cols // 2 + cols]


def _untouched(buf, view):
    rows, cols = view.shape
    at = view.storage_offset() % buf.shape[1]
    assert torch.isnan(buf[rows:]).all() and torch.isnan(buf[:, :at]).all() and torch.isnan(buf[:, at + cols:]).all()


def _within(name, got, ref, tol, norm=False):
    got = _f64(got)
    assert np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - ref) - tol
    assert (over <= 0).all(), f"{name}: {over.max():.3g} over the bound at {np.unravel_index(over.argmax(), over.shape)}"
    if norm:
        rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert rel <= HALF, f"{name}: {rel:.3g} in the 2-norm"


def _off_gu(a, w):
    return (a.shape[1] + 2) * U * np.matmul(np.abs(a), np.abs(w))


def _check_forward(M, K, F, kind, pads=(0, 0)):
    from paper_2507_00394_amd import binding as hx

    a_buf, a = _nan(M, K, 16, 2)
    a.copy_(_draw(M, (M, K)))
    w_buf, w = _nan(K, 2 * F, 16)
    w.copy_(_draw(F, (K, 2 * F), 1.5 * K ** -0.5))
    gu_buf, gu = _nan(M, 2 * F, *pads)
    h_buf, h = _nan(M, F, *pads)
    hx.helix_gated_linear_fwd(a, w, h, gu=gu, activation=kind)
    a64, w64 = _f64(a), _f64(w)
    ref, ref_gu = R.gated_fwd_ref(a64, w64, kind)
    off = _off_gu(a64, w64)
    _within("gu", gu, ref_gu, HALF * (np.abs(ref_gu) + off) + off, norm=True)
    g, u = np.split(ref_gu, 2, 1)
    og, ou = np.split(off, 2, 1)
    value = np.abs(R.activation_ref(g, kind)[0])
    off = 1.13 * (np.abs(u) + ou) * og + (value + 1.13 * og) * ou + 16 * U * np.abs(g * u)
    _within("h", h, ref, HALF * (np.abs(ref) + off) + off, norm=True)
    _untouched(h_buf, h)
    _untouched(gu_buf, gu)
    alone = torch.full((M, F), NAN, dtype=torch.bfloat16, device="cuda")
    hx.helix_gated_linear_fwd(a, w, alone, activation=kind)
    assert torch.equal(alone, h)
    return a, w, gu


def _check_backward(M, K, F, kind, a, w, gu, pads=(0, 0)):
    from paper_2507_00394_amd import binding as hx

    dh_buf, dh = _nan(M, F, 16, 1)
    dh.copy_(_draw(K, (M, F)))
    ws = torch.full((hx.helix_gated_linear_bwd_workspace_bytes(M, K, F),), 255, dtype=torch.uint8, device="cuda")   # NaN wherever nothing is written
    a64, w64, dh64 = _f64(a), _f64(w), _f64(dh)
    for kept in (None, gu):
        da_buf, da = _nan(M, K, *pads)
        dw_buf, dw = _nan(K, 2 * F, pads[0])
        hx.helix_gated_linear_bwd(a, w, dh, da, dw, ws, gu=kept, activation=kind)
        rda, rdw, dgu = R.gated_bwd_ref(a64, w64, dh64, kind, None if kept is None else _f64(kept))
        off = (HALF + 32 * U) * np.abs(dgu)
        if kept is None:   # g and u from fp32 sums: |d dg| <= |dh| (|u| |act''| off(g) + |act'| off(u)), |act''| <= 0.8
            gu64 = np.matmul(a64, w64)
            o = _off_gu(a64, w64)
            g, u = np.split(np.abs(gu64), 2, 1)
            og, ou = np.split(o, 2, 1)
            off = off + np.concatenate([np.abs(dh64) * (0.8 * (u + ou) * og + 1.13 * ou), np.abs(dh64) * 1.13 * og], 1)
        t = np.matmul(np.abs(dgu), np.abs(w64).T) * (2 * F + 2) * U * 1.01 + np.matmul(off, np.abs(w64).T)
        _within("da", da, rda, HALF * (np.abs(rda) + t) + t, norm=True)
        t = np.matmul(np.abs(a64).T, np.abs(dgu)) * (M + 40) * U * 1.01 + np.matmul(np.abs(a64).T, off)
        _within("dw", dw, rdw, HALF * (np.abs(rdw) + t) + t, norm=True)
        _untouched(da_buf, da)
        _untouched(dw_buf, dw)


# tiles of every size, whole and cut in both directions; contractions shorter than the stages in flight; one token
SHAPES = [(1, 128, 64), (1, 256, 320), (2, 384, 64), (5, 128, 704), (9, 640, 192), (17, 256, 128), (31, 128, 64), (32, 256, 192), (33, 384, 128), (64, 128, 64), (65, 512, 448), (127, 256, 320),
          (128, 128, 1024), (257, 640, 64), (513, 256, 2112), (1000, 384, 576), (2049, 128, 1088), (4100, 128, 2112), (2077, 1280, 448)]


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", SHAPES)
def test_gated(M, K, F, kind):
    a, w, gu = _check_forward(M, K, F, kind, pads=(16, 3))
    _check_backward(M, K, F, kind, a, w, gu, pads=(32, 1))


def test_weight_gradient_in_parts():
    """So many tokens, none of them dividing anything, that the weight gradient's contraction is cut into parts."""
    M, K, F = 4100, 256, 192
    a, w, gu = _check_forward(M, K, F, "silu")
    _check_backward(M, K, F, "silu", a, w, gu)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_large_arguments(kind):
    """Projections of hundreds: the exponentials run out of range without an infinity or NaN in the results."""
    from paper_2507_00394_amd import binding as hx

    M, K, F = 96, 128, 64
    a, w, dh = _draw(1, (M, K), 30.0), _draw(2, (K, 2 * F)), _draw(3, (M, F))
    h, gu = torch.empty(M, F, dtype=torch.bfloat16, device="cuda"), torch.empty(M, 2 * F, dtype=torch.bfloat16, device="cuda")
    hx.helix_gated_linear_fwd(a, w, h, gu=gu, activation=kind)
    ref, _ = R.gated_fwd_ref(_f64(a), _f64(w), kind)
    assert np.abs(_f64(gu)).max() > 500
    assert np.linalg.norm(_f64(h) - ref) <= HALF * np.linalg.norm(ref)
    _check_backward(M, K, F, kind, a, w, gu)


def test_bad_values_stay_in_their_rows():
    from paper_2507_00394_amd import binding as hx

    for M, K, F in ((1000, 256, 192), (70, 128, 64), (5, 256, 128)):
        a, w = _draw(1, (M, K)), _draw(2, (K, 2 * F), 0.1)
        a[M // 2, 3] = NAN
        a[M - 1, K - 1] = float("inf")
        h, gu = torch.empty(M, F, dtype=torch.bfloat16, device="cuda"), torch.empty(M, 2 * F, dtype=torch.bfloat16, device="cuda")
        hx.helix_gated_linear_fwd(a, w, h, gu=gu)
        good = torch.ones(M, dtype=torch.bool, device="cuda")
        good[[M // 2, M - 1]] = False
        assert torch.isfinite(h[good]).all() and torch.isfinite(gu[good]).all() and torch.isnan(h[M // 2]).all() and not torch.isfinite(gu[M - 1]).any()
        da, dw = torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(K, 2 * F, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F), dtype=torch.uint8, device="cuda")
        hx.helix_gated_linear_bwd(a, w, _draw(4, (M, F)), da, dw, ws)
        assert torch.isfinite(da[good]).all() and torch.isnan(da[M // 2]).all()


def _step(a, w, dh, out, kind):
    from paper_2507_00394_amd import binding as hx

    h, gu, da, dw, da2, dw2, ws = out
    hx.helix_gated_linear_fwd(a, w, h, gu=gu, activation=kind)
    hx.helix_gated_linear_bwd(a, w, dh, da, dw, ws, gu=gu, activation=kind)
    hx.helix_gated_linear_bwd(a, w, dh, da2, dw2, ws, activation=kind)


def _buffers(M, K, F):
    from paper_2507_00394_amd import binding as hx

    new = lambda *s: torch.full(s, NAN, dtype=torch.bfloat16, device="cuda")
    return [new(M, F), new(M, 2 * F), new(M, K), new(K, 2 * F), new(M, K), new(K, 2 * F),
            torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(M, K, F), dtype=torch.uint8, device="cuda")]


@pytest.mark.parametrize("M,K,F", [(3, 256, 192), (300, 384, 320), (4500, 256, 2048)])
def test_replays_streams_and_runs_agree_bit_for_bit(M, K, F):
    a, w, dh = _draw(1, (M, K)), _draw(2, (K, 2 * F), 0.05), _draw(3, (M, F))
    want = _buffers(M, K, F)
    _step(a, w, dh, want, "silu")
    got = _buffers(M, K, F)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(a, w, dh, got, "silu")
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want[:6], got[:6]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(a, w, dh, got, "silu")
    for _ in range(3):
        for t in got:
            t.fill_(255 if t.dtype == torch.uint8 else NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want[:6], got[:6]))


def test_the_framework_runs_it_as_the_linear_layer_does():
    """gu is what helix_qkv_linear_fwd makes of a and w; its backward takes dgu as the gated backward does inside."""
    from paper_2507_00394_amd import binding as hx

    M, K, F = 320, 256, 192
    bits = I.linear_case_bits(77, M, K, 2 * F)
    a, w = (torch.from_numpy(bits[t].view(np.int16)).cuda().view(torch.bfloat16) for t in ("a", "w"))
    h, gu, same = (torch.empty(M, n, dtype=torch.bfloat16, device="cuda") for n in (F, 2 * F, 2 * F))
    hx.helix_gated_linear_fwd(a, w, h, gu=gu)
    hx.helix_qkv_linear_fwd(a, w, same)
    _within("gu", gu, _f64(same), 2 * HALF * np.abs(_f64(same)) + 2 * _off_gu(_f64(a), _f64(w)))


def test_the_pitch_of_a_single_row_counts_for_nothing():
    """One token taken from a buffer whose rows are an odd number of elements apart: there is no next row."""
    from paper_2507_00394_amd import binding as hx

    K, F = 256, 192
    w = _draw(1, (K, 2 * F), K ** -0.5)
    row = lambda n: torch.as_strided(torch.zeros(n, dtype=torch.bfloat16, device="cuda"), (1, n), (n + 3, 1))
    results = []
    for new in (row, lambda n: torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")):
        a, dh, h, gu, da, dw = new(K), new(F), new(F), new(2 * F), new(K), torch.empty_like(w)
        a.copy_(_draw(2, (1, K)))
        dh.copy_(_draw(3, (1, F)))
        hx.helix_gated_linear_fwd(a, w, h, gu=gu)
        hx.helix_gated_linear_bwd(a, w, dh, da, dw, torch.empty(hx.helix_gated_linear_bwd_workspace_bytes(1, K, F), dtype=torch.uint8, device="cuda"), gu=gu)
        results.append((h, gu, da, dw))
    assert all(torch.equal(x, y) and y.abs().max() > 0 for x, y in zip(*results))


# a wave's share of the contraction: none, less than what it has on its way, exactly that, twice that and some; token blocks whole and cut; neighbouring workgroups on either side of
# the last group of sixteen; the widest that is left to the few-rows kernel and the narrowest that is not
@pytest.mark.parametrize("M,K,F", [(1, 1536, 64), (4, 2048, 576), (15, 1664, 128), (16, 3200, 192), (17, 2944, 64), (32, 4736, 128), (29, 384, 1088), (16, 128, 8192), (3, 256, 8256), (32, 128, 8320)])
def test_few_rows(M, K, F):
    a, w, gu = _check_forward(M, K, F, "silu")
    _check_backward(M, K, F, "silu", a, w, gu)
