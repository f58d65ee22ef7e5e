"""Definitions, in float64 numpy, of the operators of a fine-tuning step (test
infrastructure, sharing no code with the package):

  * matrices in 8-bit floating point (e4m3) with a scale 2^(s - 127) for each
    block of 128 columns and 1 or 128 rows, and the products of such a weight;
  * cross entropy of softmax(X W^T) against labels, with its gradients;
  * dropout drawn from Philox4x64-10.
"""
from __future__ import annotations

import numpy as np

from .dropout_rng import keep_threshold, philox4x64_10

# The 127 magnitudes of e4m3 by code: subnormals f 2^-9, then (1 + f/8) 2^(e - 7).
E4M3 = np.array([f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)][:127])


def _f64(bits: np.ndarray) -> np.ndarray:
    return (np.ascontiguousarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def fp8_nearest(y: np.ndarray) -> np.ndarray:
    """Codes (0..255) of values already divided by their scale, at most 448 in size:
    the nearest magnitude, of two equally near the even code; the sign above."""
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(E4M3, mag), 1, 126)     # E4M3[hi - 1] <= mag <= E4M3[hi] (or mag beyond either end)
    lo = hi - 1
    below, above = mag - E4M3[lo], E4M3[hi] - mag
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return code + 128 * np.signbit(y)


def fp8_scale_bytes(x: np.ndarray, block_rows: int) -> np.ndarray:
    """The scale byte of every (row group, block) of x [rows, k]."""
    rows, k = x.shape
    groups, blocks = -(-rows // block_rows), -(-k // 128)
    out = np.zeros((groups, blocks), np.int64)
    for i in range(groups):
        for b in range(blocks):
            v = x[i * block_rows:(i + 1) * block_rows, 128 * b:128 * b + 128]
            if not np.isfinite(v).all():
                out[i, b] = 255
                continue
            top, s = np.abs(v).max(), 0
            if top > 0:                                   # the smallest s whose largest value reaches the top
                s = max(0, int(np.floor(np.log2(top))) - 9 + 127)
                while 448.0 * 2.0 ** (s - 127) < top:
                    s += 1
            out[i, b] = s
    return out


def fp8_scale_place(i, b, rows: int):
    """Byte of the scale of row i, block b, of activations."""
    return (b * (-(-rows // 64)) + i // 64) * 64 + (i % 16) * 4 + (i // 16) % 4


def fp8_encode(bits: np.ndarray, block_rows: int):
    """bf16 patterns [rows, k] -> codes [rows, 128 ceil(k/128)] and scales, as bytes."""
    x = _f64(bits)
    rows, k = x.shape
    blocks = -(-k // 128)
    s = fp8_scale_bytes(x, block_rows)
    per_row = np.repeat(s, block_rows, axis=0)[:rows]
    wide = np.zeros((rows, blocks * 128))
    wide[:, :k] = x
    wide = wide.reshape(rows, blocks, 128)
    bad = (per_row == 255)[:, :, None]
    unit = 2.0 ** (np.where(per_row == 255, 127, per_row) - 127.0)
    codes = np.where(bad, 0, fp8_nearest(np.where(bad, 0.0, wide) / unit[:, :, None]))
    if block_rows == 128:
        scales = s.astype(np.uint8).reshape(-1)
    else:
        scales = np.zeros(64 * -(-rows // 64) * blocks, np.uint8)
        i, b = np.indices((rows, blocks))
        scales[fp8_scale_place(i, b, rows)] = s
    return codes.astype(np.uint8).reshape(rows, -1), scales


def fp8_decode(codes: np.ndarray, scales: np.ndarray, k: int, block_rows: int) -> np.ndarray:
    """The float64 values [rows, k] that codes and scales stand for."""
    rows, blocks = codes.shape[0], codes.shape[1] // 128
    mag = np.append(E4M3, np.nan)[codes.astype(np.int64) % 128]
    value = np.where(codes < 128, mag, -mag)
    i, b = np.indices((rows, blocks))
    s = scales[fp8_scale_place(i, b, rows)] if block_rows == 1 else scales.reshape(-1, blocks)[i // 128, b]
    unit = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return (value.reshape(rows, blocks, 128) * unit[:, :, None]).reshape(rows, -1)[:, :k]


# ---- cross entropy -------------------------------------------------------------
def xent(x: np.ndarray, w: np.ndarray, labels: np.ndarray, dloss: np.ndarray):
    """loss [rows], G [rows, vocab], dX, dW; a label outside the vocabulary is none."""
    z = x @ w.T
    vocab = w.shape[0]
    known = (labels >= 0) & (labels < vocab)
    top = z.max(axis=1, keepdims=True)
    e = np.exp(z - top)
    total = e.sum(axis=1, keepdims=True)
    p = e / total
    rows = np.arange(len(labels))
    y = np.where(known, labels, 0)
    rest = e.copy()
    rest[rows, y] = 0.0
    rest = rest.sum(axis=1) / total[:, 0]                 # 1 - p_y without the subtraction
    loss = np.where(known, np.where(rest < 0.5, -np.log1p(-np.minimum(rest, 0.5)), np.log(total[:, 0]) + top[:, 0] - z[rows, y]), 0.0)
    g = p.copy()
    g[rows, y] = -rest
    g = np.where(known[:, None], g * dloss[:, None], 0.0)
    return loss, g, g @ w, g.T @ np.where(known[:, None], x, 0.0)


# ---- dropout ---------------------------------------------------------------------
def dropout_draws(seed: int, offset: int, count: int) -> np.ndarray:
    """The 16-bit draws of elements 0 .. count - 1."""
    out = np.zeros(-(-count // 16) * 16, np.int64)
    for t in range(-(-count // 16)):
        ctr = int(offset) + t
        words = philox4x64_10((ctr & (2 ** 64 - 1), ctr >> 64, 0, 0), (int(seed), 0))
        for e in range(16):
            out[16 * t + e] = (words[e // 4] >> (16 * (e % 4))) & 0xFFFF
    return out[:count]


def dropout_kept(seed: int, offset: int, p: float, shape) -> np.ndarray:
    return (dropout_draws(seed, offset, int(np.prod(shape))) < keep_threshold(p)).reshape(shape)
