"""fp64 statement of the 8-bit layers around the expanded projection: e4m3 codes with a scale for each block of 128, the
root-mean-square norm in front of them, the products of them.

E4M3 (OCP 8-bit floating point): sign, 4 exponent bits of bias 7, 3 mantissa bits, largest value 448 = 1.75 * 2^8, smallest
normal 2^-6, subnormals in steps of 2^-9, no infinities.
"""
from __future__ import annotations

import numpy as np

FP8_BLOCK = 128
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def e4m3_step(v: np.ndarray) -> np.ndarray:
    """Distance of neighbouring e4m3 values around |v| (at a power of two, the one above it)."""
    _, p = np.frexp(np.abs(np.asarray(v, dtype=np.float64)))          # |v| = f 2^p, f in [0.5, 1)
    return np.ldexp(1.0, np.clip(p - 1, -6, 8) - 3)


def e4m3_round(v: np.ndarray) -> np.ndarray:
    """The e4m3 value nearest to v, ties to the even code, saturating at +-448 (as float64)."""
    v = np.asarray(v, dtype=np.float64)
    step = e4m3_step(v)
    return np.clip(np.rint(v / step) * step, -E4M3_MAX, E4M3_MAX)


def _scale(amax: np.ndarray) -> np.ndarray:
    return np.where(amax == 0, 1.0, np.maximum(amax / E4M3_MAX, SCALE_MIN))


def _whole(v: np.ndarray, rows: int) -> np.ndarray:
    T, d = v.shape
    return np.pad(v, ((0, -T % rows), (0, -d % FP8_BLOCK)))


def fp8_quotients(v: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """[T, d] -> (v / scale, padded with zeros to whole groups, before the rounding to e4m3; scales [T, groups])."""
    p = _whole(np.asarray(v, dtype=np.float64), 1)
    g = p.reshape(p.shape[0], -1, FP8_BLOCK)
    s = _scale(np.abs(g).max(axis=2))
    return (g / s[:, :, None]).reshape(p.shape), s


def fp8_quotients_weights(w: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """[N, d] -> (w / scale of its 128 x 128 block, [N, whole groups]; scales [ceil(N / 128), groups])."""
    p = _whole(np.asarray(w, dtype=np.float64), FP8_BLOCK)
    b = p.reshape(p.shape[0] // FP8_BLOCK, FP8_BLOCK, -1, FP8_BLOCK)
    s = _scale(np.abs(b).max(axis=(1, 3)))
    return (b / s[:, None, :, None]).reshape(p.shape)[: w.shape[0]], s


def rmsnorm(h: np.ndarray, weight: np.ndarray, eps: float) -> np.ndarray:
    h = np.asarray(h, dtype=np.float64)
    mean = np.mean(h * h, axis=1, keepdims=True) + eps
    return np.divide(h, np.sqrt(mean), out=np.zeros_like(h), where=mean > 0) * np.asarray(weight, dtype=np.float64)


def gemm_fp8(qx: np.ndarray, sx: np.ndarray, qw: np.ndarray, sw: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """Values of codes [T, K] and [N, K] with their scales -> (product [T, N], sum of the terms' magnitudes)."""
    x = np.asarray(qx, np.float64) * np.repeat(np.asarray(sx, np.float64), FP8_BLOCK, axis=1)
    w = np.asarray(qw, np.float64) * np.repeat(np.repeat(np.asarray(sw, np.float64), FP8_BLOCK, axis=0)[: len(qw)], FP8_BLOCK, axis=1)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def gated(g: np.ndarray, u: np.ndarray) -> np.ndarray:
    """silu(g) * u."""
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u
