"""Plain fp64 references of the operators around the attention stage: dropout from a counter-based generator with the
residual sum, layer norm, both together, and their gradients.

TEST INFRASTRUCTURE ONLY -- see the package docstring.

    keep_ij = (16 bits of Philox4x32-10 for row first_row + i, column j) >= cut,   cut = round(p * 2^16)
    dropout and sum   out = r + keep * x / (1 - cut / 2^16)
    layer norm        y = (x - mean) * rstd * gamma + beta,   rstd = (var + eps)^-1/2

Parity pins (tests marked "not gpu"): the generator's published known answers and its arithmetic in Python integers,
the frequency of what is kept, scalar loops, and central finite differences of every gradient.
"""
from __future__ import annotations

import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85   # Salmon et al. 2011: multipliers and the key's increments


def philox4x32(counter, key, rounds=10):
    """Four 32-bit words (uint64 arrays) of the block `counter` (four words) under `key` (two words)."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) for w in key]
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        p0, p1 = np.uint64(M0) * c[0], np.uint64(M1) * c[2]
        c = [(p1 >> shift) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> shift) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def dropout_cut(p) -> int:
    return min(int(np.rint(float(np.float32(p)) * 65536)), 65535)


def dropout_keep(seed, offset, first_row, M, E, p):
    """[M, E] truth values."""
    seed, offset = int(seed) % 2 ** 64, int(offset) % 2 ** 64
    chunk = np.arange((E + 7) // 8, dtype=np.uint64)[None, :]
    row = np.arange(first_row, first_row + M, dtype=np.uint64)[:, None]
    shape = np.broadcast_shapes(chunk.shape, row.shape)
    words = philox4x32([np.broadcast_to(chunk, shape), np.broadcast_to(row, shape), np.full(shape, offset % 2 ** 32), np.full(shape, offset >> 32)],
                       (seed % 2 ** 32, seed >> 32))
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1)
    return halves.reshape(M, -1)[:, :E] >= dropout_cut(p)


def dropout_add_ref(x, r, p, keep):
    v = np.where(keep, np.asarray(x, np.float64) / (1 - dropout_cut(p) / 65536), 0.0)
    return v if r is None else v + np.asarray(r, np.float64)


def layer_norm_fwd_ref(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64), mean, rstd


def layer_norm_bwd_ref(dy, x, gamma, mean, rstd):
    """dx, dgamma, dbeta from the forward's statistics."""
    dy, x, gamma, mean, rstd = (np.asarray(t, np.float64) for t in (dy, x, gamma, mean, rstd))
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


# ---------------------------------------------------------------- gated feed-forward projections
#     [g u] = a w,  h = act(g) * u;   dg = dh * u * act'(g),  du = dh * act(g),  da = [dg du] w^T,  dw = a^T [dg du]
def activation_ref(g, kind):
    """act(g), act'(g)."""
    g = np.asarray(g, np.float64)
    if kind == "silu":
        s = 0.5 * (1 + np.tanh(0.5 * g))
        return g * s, s + g * s * (1 - s)
    from scipy.special import erfc

    P = 0.5 * erfc(-g / np.sqrt(2))   # 1 + erf has no correct digit left below -8
    return g * P, P + g * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)


def gated_fwd_ref(a, w, kind):
    """h, gu."""
    gu = np.matmul(np.asarray(a, np.float64), np.asarray(w, np.float64))
    g, u = np.split(gu, 2, 1)
    return activation_ref(g, kind)[0] * u, gu


def gated_bwd_ref(a, w, dh, kind, gu=None):
    """da, dw, dgu; gu: the projections to start from (None: those of a and w)."""
    a, w, dh = (np.asarray(t, np.float64) for t in (a, w, dh))
    g, u = np.split(np.matmul(a, w) if gu is None else np.asarray(gu, np.float64), 2, 1)
    value, slope = activation_ref(g, kind)
    dgu = np.concatenate([dh * u * slope, dh * value], 1)
    return np.matmul(dgu, w.T), np.matmul(a.T, dgu), dgu
