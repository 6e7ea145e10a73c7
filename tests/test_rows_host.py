"""Row-wise operators on the host (no GPU): bad arguments are refused before any HIP call, by the library and by the binding."""
import ctypes

import pytest
import torch

from paper_2507_00394_amd import binding as hx

P, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10001)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not hx.LIB_PATH.exists():
        from paper_2507_00394_amd import build

        build.build()
    return hx.lib()


def test_dropout_add_refusals(L):
    def fwd(x=P, ldx=64, r=P, ldr=64, out=P, ldo=64, M=8, E=64, kind=0, p=0.1, rng=P, first=0):
        return L.helix_dropout_add_fwd(x, ldx, r, ldr, out, ldo, M, E, kind, p, rng, first, None)

    assert fwd(x=None) == 1 and fwd(out=None) == 1 and fwd(rng=None) == 1
    assert fwd(kind=3) == 10 and fwd(kind=-1) == 10
    assert fwd(x=ODD) == 4 and fwd(r=ODD) == 4 and fwd(out=ODD) == 4 and fwd(rng=ctypes.c_void_p(0x10004)) == 4
    assert fwd(kind=2, x=ctypes.c_void_p(0x10002)) == 4
    assert fwd(M=0) == 2 and fwd(E=0) == 2 and fwd(M=-1) == 2 and fwd(E=(1 << 30) + 1, ldx=1 << 31, ldr=1 << 31, ldo=1 << 31) == 2
    assert fwd(ldx=63) == 8 and fwd(ldr=63) == 8 and fwd(ldo=0) == 8 and fwd(ldo=1 << 40) == 8 and fwd(ldx=1 << 37) == 8
    assert fwd(ldo=(1 << 63) - 1) == 8
    assert fwd(p=-0.1) == 11 and fwd(p=1.0) == 11 and fwd(p=NAN) == 11 and fwd(p=INF) == 11
    assert fwd(first=-1) == 2 and fwd(first=(1 << 32) - 7) == 2
    bwd = lambda g=P, dx=P, p=0.1, rng=P, ld=64: L.helix_dropout_add_bwd(g, ld, dx, 64, 8, 64, 0, p, rng, 0, None)
    assert bwd(g=None) == 1 and bwd(dx=None) == 1 and bwd(rng=None) == 1 and bwd(p=1.5) == 11 and bwd(ld=8) == 8


def test_layer_norm_refusals(L):
    def fwd(x=P, ldx=64, g=P, b=P, y=P, ldy=64, mean=P, rstd=P, M=8, E=64, kind=0, eps=1e-5):
        return L.helix_layer_norm_fwd(x, ldx, g, b, y, ldy, mean, rstd, M, E, kind, eps, None)

    assert fwd(x=None) == 1 and fwd(g=None) == 1 and fwd(b=None) == 1 and fwd(y=None) == 1
    assert fwd(g=ctypes.c_void_p(0x10002)) == 4 and fwd(mean=ODD) == 4 and fwd(rstd=ctypes.c_void_p(0x10002)) == 4 and fwd(y=ODD) == 4
    assert fwd(M=0) == 2 and fwd(E=0) == 2 and fwd(E=16385, ldx=16385, ldy=16385) == 2
    assert fwd(ldx=63) == 8 and fwd(ldy=63) == 8 and fwd(kind=7) == 10
    assert fwd(eps=0.0) == 12 and fwd(eps=-1.0) == 12 and fwd(eps=NAN) == 12 and fwd(eps=INF) == 12

    need = hx.helix_layer_norm_bwd_workspace_bytes(8, 64)
    assert need >= 2 * 64 * 4 and need % 256 == 0

    def bwd(dy=P, x=P, mean=P, rstd=P, dx=P, dg=P, db=P, ws=P, n=need, ld=64, M=8, E=64):
        return L.helix_layer_norm_bwd(dy, ld, x, 64, P, mean, rstd, dx, 64, dg, db, ws, n, M, E, 0, None)

    assert all(bwd(**{k: None}) == 1 for k in ("dy", "x", "mean", "rstd", "dx", "dg", "db", "ws"))
    assert bwd(ws=ctypes.c_void_p(0x10010)) == 4 and bwd(n=need - 1) == 6 and bwd(ld=60) == 8 and bwd(M=0) == 2

    def both(x=P, r=P, s=P, y=P, p=0.1, rng=P, first=0, eps=1e-5, lds=64):
        return L.helix_dropout_add_layer_norm_fwd(x, 64, r, 64, s, lds, P, P, y, 64, P, P, 8, 64, 0, p, rng, first, eps, None)

    assert both(x=None) == 1 and both(r=None) == 1 and both(s=None) == 1 and both(y=None) == 1 and both(rng=None) == 1
    assert both(p=1.0) == 11 and both(first=-1) == 2 and both(eps=0.0) == 12 and both(lds=63) == 8

    def both_bwd(dy=P, ds=P, s=P, dx=P, dr=P, ws=P, n=need, p=0.1, rng=P, ldds=64):
        return L.helix_dropout_add_layer_norm_bwd(dy, 64, ds, ldds, s, 64, P, P, P, dx, 64, dr, 64, P, P, ws, n, 8, 64, 0, p, rng, 0, None)

    assert both_bwd(dy=None) == 1 and both_bwd(s=None) == 1 and both_bwd(dx=None) == 1 and both_bwd(dr=None) == 1 and both_bwd(ws=None) == 1
    assert both_bwd(rng=None) == 1 and both_bwd(ds=ODD) == 4 and both_bwd(ldds=63) == 8 and both_bwd(n=0) == 6 and both_bwd(p=NAN) == 11


def test_workspace_bytes(L):
    assert hx.helix_layer_norm_bwd_workspace_bytes(0, 64) == 0 and hx.helix_layer_norm_bwd_workspace_bytes(4, 0) == 0
    assert hx.helix_layer_norm_bwd_workspace_bytes(4, 16385) == 0
    for M in (1, 3, 100, 5000, 131072, 2 ** 31 - 1):
        for E in (1, 64, 1000, 4096, 16384):
            n = hx.helix_layer_norm_bwd_workspace_bytes(M, E)
            assert 8 * E <= n <= 256 * 1024 * 2 * 4 * E and n % 256 == 0
    assert hx.helix_layer_norm_bwd_workspace_bytes(1, 4096) == 2 * 4096 * 4     # one row leaves one slab


def test_new_statuses_have_names(L):
    assert len({hx.status_string(s) for s in range(13)}) == 13


def test_binding_refuses(L):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    f = torch.zeros(64)
    with pytest.raises(ValueError):
        hx.helix_layer_norm_fwd(x, f, f, x, torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError):
        hx.helix_dropout_add_fwd(x, None, x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        hx.helix_dropout_add_bwd(x.double(), x, 0.1, None)


def test_lengths_of_more_than_32_bits_are_refused(L, monkeypatch):
    """The library's lengths have 32 bits: what is longer must not arrive there as what is left of it."""
    long = 2 ** 32 + 3
    assert hx.helix_layer_norm_bwd_workspace_bytes(long, 64) == 0 and hx.helix_layer_norm_bwd_workspace_bytes(4, 2 ** 32 + 64) == 0
    for shape in ((2 ** 32 + 4, 256, 128), (4, 2 ** 32 + 256, 128), (4, 256, 2 ** 32 + 128)):
        assert hx.helix_gated_linear_bwd_workspace_bytes(*shape) == 0
    monkeypatch.setattr(hx, "_current", lambda t, stream: -1)     # host memory stands for the device's: nothing gets as far as a kernel
    monkeypatch.setattr(hx, "_stream", lambda stream: None)
    for M, E in ((long, 1), (1, long)):
        x = torch.empty_strided((M, E), (1, 1) if E == 1 else (E, 1), dtype=torch.float16)   # never touched, so it takes no memory
        with pytest.raises(hx.HelixStatusError) as e:
            hx.helix_dropout_add_fwd(x, None, x, 0.0, None)
        assert e.value.status == 2
        with pytest.raises(hx.HelixStatusError) as e:
            hx.helix_dropout_add_bwd(x, x, 0.0, None)
        assert e.value.status == 2
    x, rng = torch.zeros(4, 64), torch.zeros(2, dtype=torch.int64)
    for first in (-1, 2 ** 32, 2 ** 64, 2 ** 64 - 1, -2 ** 64):
        with pytest.raises(hx.HelixStatusError) as e:
            hx.helix_dropout_add_fwd(x, None, x, 0.5, rng, first_row=first)
        assert e.value.status == 2
