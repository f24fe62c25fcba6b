"""Plain 64-bit implementations (numpy) of the dense operators: matrix product with its epilogue, group norm with an activation,
dropout from the Philox generator.

TEST INFRASTRUCTURE ONLY, like the rest of this package: written from the definitions, sharing no code with the product.  Every
function takes and returns float64 arrays that hold the stored values exactly.
"""
from __future__ import annotations

import math

import numpy as np
from scipy import special

M32 = np.uint64(0xFFFFFFFF)


def philox(seed: int, call: int, first_block: int, blocks: int) -> np.ndarray:
    """Words [blocks, 4] of Philox 4x32-10 with key = seed and counters (first_block + i, call)."""
    i = np.arange(blocks, dtype=np.uint64) + np.uint64(first_block)
    seed, call = seed % 2 ** 64, call % 2 ** 64
    c = [i & M32, i >> np.uint64(32), np.full_like(i, call % 2 ** 32), np.full_like(i, call >> 32)]
    k = [seed % 2 ** 32, seed >> 32]
    for _ in range(10):
        a = c[0] * np.uint64(0xD2511F53)
        b = c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & M32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & M32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, axis=1)


def keep(shape, p: float, seed: int, call: int) -> np.ndarray:
    """Truth of `element stays`, elements in the order of memory."""
    n = int(np.prod(shape))
    least = math.floor(float(np.float32(p)) * 2.0 ** 32)
    return (philox(seed, call, 0, -(-n // 4)).reshape(-1)[:n] >= np.uint64(least)).reshape(shape)


def drop(v: np.ndarray, p: float, rng) -> np.ndarray:
    if not p:
        return v
    return np.where(keep(v.shape, p, *rng), v * (1.0 / (1.0 - float(np.float32(p)))), 0.0)


def act(z: np.ndarray, name: str) -> np.ndarray:
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return z * special.ndtr(z)
    if name == "silu":
        return z * special.expit(z)
    return z


def slope(z: np.ndarray, name: str) -> np.ndarray:
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return special.ndtr(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = special.expit(z)
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear_fwd(x, w, bias=None, residual=None, name="none", p=0.0, rng=None):
    """-> (out, pre)"""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    out = drop(act(z, name), p, rng)
    return (out if residual is None else residual + out), z


def linear_dz(dout, pre, name="none", p=0.0, rng=None):
    dz = drop(dout, p, rng)
    return dz if name == "none" else dz * slope(pre, name)


def linear_bwd(x, w, dout, pre=None, name="none", p=0.0, rng=None):
    """-> dict(dx, dweight, dbias)"""
    dz = linear_dz(dout, pre, name, p, rng)
    return {"dx": dz @ w, "dweight": dz.T @ x, "dbias": dz.sum(0)}


def _groups(v, G):
    B, N, C = v.shape
    return v.reshape(B, N, G, C // G)


def norm_fwd(x, gamma, beta, G, eps, name="none"):
    """-> (out, mean [B,G], rstd [B,G])"""
    v = _groups(x, G)
    mean = v.mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3)) + eps)
    z = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    if gamma is not None:
        z = z * gamma + beta
    return act(z, name), mean, rstd


def norm_bwd(x, gamma, beta, mean, rstd, dout, G, name="none"):
    """-> dict(dx, dgamma, dbeta)"""
    r = rstd[:, None, :, None]
    xhat = ((_groups(x, G) - mean[:, None, :, None]) * r).reshape(x.shape)
    dz = dout * slope(xhat if gamma is None else xhat * gamma + beta, name)
    dh = _groups(dz if gamma is None else dz * gamma, G)
    xh = _groups(xhat, G)
    dx = r * (dh - dh.mean(axis=(1, 3), keepdims=True) - xh * (dh * xh).mean(axis=(1, 3), keepdims=True))
    return {"dx": dx.reshape(x.shape), "dgamma": (dz * xhat).sum(axis=(0, 1)), "dbeta": dz.sum(axis=(0, 1))}
