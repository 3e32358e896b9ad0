"""The 8-bit form of activations and the operators on it in 64 bits, from their definitions (numpy, no GPU)."""
from __future__ import annotations

import math

import numpy as np

import oracle

GROUP = 32
NONE, RELU, SILU, GELU = 0, 1, 2, 3
_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def groups(cols: int) -> int:
    return -(-cols // GROUP)


def unit(byte: int) -> float:
    return math.nan if byte == 255 else 0.0 if byte == 0 else math.ldexp(1.0, byte - 127)


def byte_of(amax: float) -> int:
    """Byte of a group with this largest magnitude."""
    if not math.isfinite(amax):
        return 255
    e = -120
    while e < 121 and amax > math.ldexp(127.0, e):
        e += 1
    return e + 127


def encode(x: np.ndarray, random=None):
    """(codes, scales) of x [rows, cols]; random = (seed, stream_id, which) for the rounding at random."""
    rows, cols = x.shape
    x32 = x.astype(np.float32)
    codes = np.zeros((rows, cols), np.int8)
    scales = np.zeros((rows, groups(cols)), np.uint8)
    words = {}
    for r in range(rows):
        for g in range(groups(cols)):
            v = x32[r, g * GROUP:(g + 1) * GROUP]
            b = byte_of(float(np.max(np.abs(v.astype(np.float64)))) if np.all(np.isfinite(v)) else math.inf)
            scales[r, g] = b
            if b == 255:
                continue
            t = (v * np.float32(math.ldexp(1.0, 127 - b))).astype(np.float32)
            t = np.clip(t, np.float32(-127), np.float32(127))
            if random is None:
                q = np.rint(t)
            else:
                seed, stream, which = random
                f = np.floor(t)
                u = np.zeros(len(v), np.float32)
                for j in range(len(v)):
                    i = r * cols + g * GROUP + j
                    if i // 4 not in words:
                        words[i // 4] = oracle.philox4x32_10([(i // 4) & 0xFFFFFFFF, (i // 4) >> 32, which, stream],
                                                             [seed & 0xFFFFFFFF, seed >> 32])
                    u[j] = np.float32(int(words[i // 4][i % 4]) >> 8)
                q = f + (u < ((t - f).astype(np.float32) * np.float32(2 ** 24)).astype(np.float32))
            codes[r, g * GROUP:(g + 1) * GROUP] = q.astype(np.int64)
    return codes, scales


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    units = np.array([unit(int(b)) for b in scales.reshape(-1)]).reshape(scales.shape)
    return codes.astype(np.float64) * np.repeat(units, GROUP, axis=1)[:, :codes.shape[1]]


def value(act: int, z: np.ndarray) -> np.ndarray:
    if act == RELU:
        return np.where(z > 0, z, np.where(np.isnan(z), z, 0.0))
    if act == SILU:
        return z / (1 + np.exp(-z))
    if act == GELU:
        return 0.5 * z * _erfc(-z / math.sqrt(2))
    return z.copy()


def slope(act: int, z: np.ndarray) -> np.ndarray:
    if act == RELU:
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
    if act == SILU:
        s = 1 / (1 + np.exp(-z))
        return s + z * s * (1 - s)
    if act == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def group_stats(x: np.ndarray, G: int, eps: float):
    N, P, C = x.shape
    v = x.reshape(N, P, G, C // G) if C else x.reshape(N, P, G, 0)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1 / np.sqrt(var + eps)


def wide(s: np.ndarray, C: int) -> np.ndarray:
    return np.repeat(s, C // s.shape[1], axis=1)[:, None, :]


def group_norm_backward(dy, x, mean, rstd, gamma, beta, G, act):
    N, P, C = x.shape
    xh = (x - wide(mean, C)) * wide(rstd, C)
    dz = dy * slope(act, gamma * xh + beta)
    gz = gamma * dz
    m1 = gz.reshape(N, P, G, C // G).mean(axis=(1, 3))
    m2 = (gz * xh).reshape(N, P, G, C // G).mean(axis=(1, 3))
    dx = wide(rstd, C) * (gz - wide(m1, C) - xh * wide(m2, C))
    return dx, (dz * xh).sum(axis=(0, 1)), dz.sum(axis=(0, 1)), xh, dz
