"""Gated projections on the host (no GPU): bad arguments are refused before any HIP call, by the library and by the binding."""
import ctypes

import pytest
import torch

from paper_2507_00394_amd import binding as hx

P, ODD, NEAR = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10010)


@pytest.fixture(scope="module")
def L():
    if not hx.LIB_PATH.exists():
        from paper_2507_00394_amd import build

        build.build()
    return hx.lib()


def test_forward_refusals(L):
    def fwd(a=P, lda=128, w=P, ldw=128, gu=None, ldgu=0, h=P, ldh=64, M=3, K=128, F=64, act=0):
        return L.helix_gated_linear_fwd(a, lda, w, ldw, gu, ldgu, h, ldh, M, K, F, act, None)

    assert fwd(a=None) == 1 and fwd(w=None) == 1 and fwd(h=None) == 1
    assert fwd(a=ODD) == 4 and fwd(gu=ODD, ldgu=128) == 4 and fwd(h=ODD) == 4
    assert fwd(act=2) == 10 and fwd(act=-1) == 10
    assert fwd(M=0) == 2 and fwd(K=96) == 2 and fwd(F=32, ldw=128) == 2 and fwd(F=0) == 2 and fwd(F=-64) == 2 and fwd(M=2 ** 31 - 1) == 2
    assert fwd(F=2 ** 31 - 64) == 2 and fwd(F=(1 << 19) + 64) == 2 and fwd(K=(1 << 20) + 128) == 2
    assert fwd(lda=120) == 8 and fwd(lda=132) == 8 and fwd(ldw=120) == 8 and fwd(ldh=56) == 8 and fwd(gu=P, ldgu=120) == 8 and fwd(ldh=(1 << 22) + 8) == 8


def test_backward_refusals(L):
    need = hx.helix_gated_linear_bwd_workspace_bytes(3, 128, 64)

    def bwd(a=P, lda=128, w=P, gu=None, ldgu=0, dh=P, lddh=64, da=P, ldda=128, dw=P, lddw=128, ws=P, n=need, M=3, K=128, F=64, act=1):
        return L.helix_gated_linear_bwd(a, lda, w, 128, gu, ldgu, dh, lddh, da, ldda, dw, lddw, ws, n, M, K, F, act, None)

    assert all(bwd(**{k: None}) == 1 for k in ("a", "w", "dh", "da", "dw", "ws"))
    assert bwd(dh=ODD) == 4 and bwd(gu=ODD, ldgu=128) == 4 and bwd(ws=NEAR) == 4
    assert bwd(n=need - 1) == 6 and bwd(act=5) == 10 and bwd(M=0) == 2 and bwd(F=65) == 2
    assert bwd(lddh=60) == 8 and bwd(ldda=64) == 8 and bwd(lddw=64) == 8 and bwd(gu=P, ldgu=64) == 8 and bwd(lda=1 << 23) == 8


def test_workspace_bytes(L):
    # [dg du] of the rows up to a multiple of 32, behind the linear layer's w^T and partial sums
    assert hx.helix_gated_linear_bwd_workspace_bytes(33, 128, 64) == hx.helix_qkv_linear_bwd_workspace_bytes(64, 128, 128) + 64 * 128 * 2
    assert hx.helix_gated_linear_bwd_workspace_bytes(0, 128, 64) == 0 and hx.helix_gated_linear_bwd_workspace_bytes(1, 128, 63) == 0
    assert hx.helix_gated_linear_bwd_workspace_bytes(1, 100, 64) == 0 and hx.helix_gated_linear_bwd_workspace_bytes(1, 128, 2 ** 31 - 64) == 0


def test_binding_refuses(L):
    a, w, h = (torch.zeros(*s, dtype=torch.bfloat16) for s in ((4, 128), (128, 128), (4, 64)))
    with pytest.raises(ValueError):
        hx.helix_gated_linear_fwd(a, w, h)                                   # not on a device
    with pytest.raises(ValueError):
        hx.helix_gated_linear_fwd(a, w, h, activation="relu")
    with pytest.raises(ValueError):
        hx.helix_gated_linear_fwd(a, w[:, :127], h)
