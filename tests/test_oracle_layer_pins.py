"""Pins of the oracle of the operators around the attention stage (no GPU)."""
import numpy as np
import pytest

from oracle import layer_ref as R


def test_generator_known_answers():
    """The known answers published with the generator (Random123)."""
    answers = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
               ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
               ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for counter, key, want in answers:
        assert tuple(int(w) for w in R.philox4x32(counter, key)) == want


def test_generator_against_python_integers():
    rng = np.random.Generator(np.random.Philox(11))
    for _ in range(20):
        c, k = [int(v) for v in rng.integers(0, 2 ** 32, 4)], [int(v) for v in rng.integers(0, 2 ** 32, 2)]
        want = list(c)
        key = list(k)
        for _ in range(10):
            a, b = R.M0 * want[0], R.M1 * want[2]
            want = [(b >> 32) ^ want[1] ^ key[0], b % 2 ** 32, (a >> 32) ^ want[3] ^ key[1], a % 2 ** 32]
            key = [(key[0] + R.W0) % 2 ** 32, (key[1] + R.W1) % 2 ** 32]
        assert [int(w) for w in R.philox4x32(c, k)] == want


def test_keep_layout_and_frequency():
    seed, offset = -5, 2 ** 40 + 3
    keep = R.dropout_keep(seed, offset, 7, 6, 21, 0.25)
    for i in range(6):
        for j in range(21):
            words = R.philox4x32((j // 8, 7 + i, 3, 2 ** 8), (2 ** 32 - 5, 2 ** 32 - 1))
            w = int(words[(j % 8) // 2])
            assert keep[i, j] == ((w >> 16 if j % 2 else w & 0xFFFF) >= 16384)
    p = 0.1
    share = R.dropout_keep(1, 2, 0, 1000, 1000, p).mean()
    cut = R.dropout_cut(p) / 65536
    assert abs(share - (1 - cut)) < 5 * np.sqrt(cut * (1 - cut) / 1e6)
    # rows are numbered: a part of a call is the part of the mask
    assert np.array_equal(R.dropout_keep(1, 2, 4, 3, 100, p), R.dropout_keep(1, 2, 0, 9, 100, p)[4:7])


def test_layer_norm_scalar_loops():
    rng = np.random.Generator(np.random.Philox(12))
    x, gamma, beta = rng.standard_normal((4, 9)), rng.standard_normal(9), rng.standard_normal(9)
    y, mean, rstd = R.layer_norm_fwd_ref(x, gamma, beta, 1e-3)
    for i in range(4):
        m = sum(x[i]) / 9
        v = sum((t - m) ** 2 for t in x[i]) / 9
        assert mean[i] == pytest.approx(m, abs=1e-14) and rstd[i] == pytest.approx((v + 1e-3) ** -0.5, rel=1e-13)
        for j in range(9):
            assert y[i, j] == pytest.approx((x[i, j] - m) * (v + 1e-3) ** -0.5 * gamma[j] + beta[j], abs=1e-13)


def test_gradients_by_differences():
    """Central differences of L = sum(w * y) + sum(u * s) for s = r + dropout(x), y = layer norm of s."""
    rng = np.random.Generator(np.random.Philox(13))
    M, E, eps, p = 3, 11, 1e-2, 0.3
    x, r, w, u = (rng.standard_normal((M, E)) for _ in range(4))
    gamma, beta = rng.standard_normal(E), rng.standard_normal(E)
    keep = R.dropout_keep(3, 4, 0, M, E, p)

    def loss(x, r, gamma, beta):
        s = R.dropout_add_ref(x, r, p, keep)
        return (w * R.layer_norm_fwd_ref(s, gamma, beta, eps)[0]).sum() + (u * s).sum()

    s = R.dropout_add_ref(x, r, p, keep)
    _, mean, rstd = R.layer_norm_fwd_ref(s, gamma, beta, eps)
    ds, dgamma, dbeta = R.layer_norm_bwd_ref(w, s, gamma, mean, rstd)
    ds = ds + u
    grads = {0: R.dropout_add_ref(ds, None, p, keep), 1: ds, 2: dgamma, 3: dbeta}
    args = [x, r, gamma, beta]
    h = 1e-5
    for k, want in grads.items():
        for idx in np.ndindex(args[k].shape):
            a, b = [t.copy() for t in args], [t.copy() for t in args]
            a[k][idx] += h
            b[k][idx] -= h
            assert (loss(*a) - loss(*b)) / (2 * h) == pytest.approx(want[idx], rel=1e-6, abs=1e-7)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_scalar_loops_and_differences(kind):
    import math

    rng = np.random.Generator(np.random.Philox(14))
    M, K, F = 3, 5, 4
    a, w, dh = rng.standard_normal((M, K)), rng.standard_normal((K, 2 * F)), rng.standard_normal((M, F))
    act = (lambda g: g / (1 + math.exp(-g))) if kind == "silu" else (lambda g: g * 0.5 * math.erfc(-g / math.sqrt(2)))
    h, gu = R.gated_fwd_ref(a, w, kind)
    for i in range(M):
        for j in range(F):
            g, u = sum(a[i, k] * w[k, j] for k in range(K)), sum(a[i, k] * w[k, F + j] for k in range(K))
            assert h[i, j] == pytest.approx(act(g) * u, rel=1e-12, abs=1e-13) and gu[i, j] == pytest.approx(g, abs=1e-13)
    da, dw, _ = R.gated_bwd_ref(a, w, dh, kind)
    step = 1e-5
    for x, grad, loss in ((a, da, lambda t: (dh * R.gated_fwd_ref(t, w, kind)[0]).sum()), (w, dw, lambda t: (dh * R.gated_fwd_ref(a, t, kind)[0]).sum())):
        for idx in np.ndindex(x.shape):
            up, down = x.copy(), x.copy()
            up[idx] += step
            down[idx] -= step
            assert (loss(up) - loss(down)) / (2 * step) == pytest.approx(grad[idx], rel=1e-6, abs=1e-8)
    kept = R.gated_bwd_ref(a, w, dh, kind, gu=gu)
    assert np.allclose(kept[0], da, rtol=1e-13) and np.allclose(kept[1], dw, rtol=1e-13)
