"""Definitions, in float64 numpy, of the operators around the layer's output
(test infrastructure, sharing no code with the package):

  * microscaled 4-bit matrices: blocks of 32 columns with a scale 2^(s - 127),
    elements 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, and their linear layer;
  * log probability of a token, entropy and the top alternatives of a row;
  * distillation from a teacher's top logits, loss and gradient.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _f64(bits: np.ndarray) -> np.ndarray:
    """bf16 patterns (uint16) -> float64, exact."""
    return (np.ascontiguousarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ---- microscaled 4 bits -------------------------------------------------------
def mx4_nearest(y: np.ndarray) -> np.ndarray:
    """Codes (0..15) of values y already divided by their scale: the nearest
    magnitude, of two equally near the even code; the sign above."""
    mag = np.minimum(np.abs(y), 6.0)
    dist = np.abs(mag[..., None] - E2M1)
    near = dist == dist.min(axis=-1, keepdims=True)
    even = np.where(near, np.arange(8) % 2, 2)          # of the nearest, an even code first
    return np.argmin(even, axis=-1) + 8 * np.signbit(y)


def mx4_blocks(x: np.ndarray):
    """x [rows, k] float64 -> codes [rows, B, 32] and scale bytes [rows, B]."""
    rows, k = x.shape
    blocks = -(-k // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :k] = x
    v = v.reshape(rows, blocks, 32)
    finite = np.isfinite(v).all(axis=2)
    top = np.where(finite, np.abs(v).max(axis=2, where=np.isfinite(v), initial=0.0), 0.0)
    exponent = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))), -1000.0)
    scale = np.where(finite, np.maximum(0, exponent - 2 + 127), 255).astype(np.int64)
    unit = 2.0 ** (np.where(finite, scale, 127) - 127.0)
    code = np.where(finite[:, :, None], mx4_nearest(np.where(finite[:, :, None], v, 0.0) / unit[:, :, None]), 0)
    return code, scale


def mx4_scale_place(i, b, rows: int):
    """Byte of the scale of row i, block b."""
    cells = -(-rows // 64)
    return ((b // 8) * cells + i // 64) * 512 + (b % 4) * 128 + (i % 16) * 8 + (i // 16 % 4) * 2 + (b // 4) % 2


def mx4_encode(bits: np.ndarray):
    """bf16 patterns [rows, k] -> codes [rows, 128 ceil(k/256)] and scales, as bytes."""
    rows, k = bits.shape
    slabs = -(-k // 256)
    code, scale = mx4_blocks(_f64(bits))
    wide = np.zeros((rows, slabs * 256), np.int64)
    wide[:, :code.shape[1] * 32] = code.reshape(rows, -1)
    scales = np.zeros(-(-rows // 64) * slabs * 512, np.uint8)
    i, b = np.indices(scale.shape)
    scales[mx4_scale_place(i, b, rows)] = scale
    return (wide[:, 0::2] + 16 * wide[:, 1::2]).astype(np.uint8), scales


def mx4_decode(codes: np.ndarray, scales: np.ndarray, k: int) -> np.ndarray:
    """The float64 values [rows, k] that codes and scales stand for."""
    rows = codes.shape[0]
    wide = np.empty((rows, codes.shape[1] * 2), np.int64)
    wide[:, 0::2], wide[:, 1::2] = codes % 16, codes // 16
    value = E2M1[wide % 8] * np.where(wide < 8, 1.0, -1.0)
    out = np.empty((rows, k))
    for b in range(-(-k // 32)):
        s = scales[mx4_scale_place(np.arange(rows), b, rows)].astype(np.float64)
        unit = np.where(s == 255, np.nan, 2.0 ** (s - 127))
        cols = slice(32 * b, min(k, 32 * b + 32))
        out[:, cols] = value[:, cols] * unit[:, None]
    return out


def mx4_linear(x_bits: np.ndarray, codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Q(X) Q(W)^T in float64."""
    k = x_bits.shape[1]
    xc, xs = mx4_encode(x_bits)
    return mx4_decode(xc, xs, k) @ mx4_decode(codes, scales, k).T


# ---- rows of logits -----------------------------------------------------------
def log_softmax(z: np.ndarray) -> np.ndarray:
    """Of one row; -inf everywhere for a row of -inf, NaN for one with a NaN or +inf."""
    if np.isnan(z).any() or np.isposinf(z).any():
        return np.full(z.shape, np.nan)
    top = z.max()
    if np.isneginf(top):
        return np.full(z.shape, -np.inf)
    return (z - top) - np.log(np.exp(z - top).sum())


def token_logprobs(z, tokens, temperature: float, top: int):
    """z [rows, vocab] float64 -> (logp, entropy, top ids, top log probabilities)."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    logp, entropy = np.zeros(rows), np.zeros(rows)
    ids, lps = np.zeros((rows, top), np.int64), np.zeros((rows, top))
    for i in range(rows):
        lq = log_softmax(z[i] / temperature)
        p = np.exp(lq)
        entropy[i] = -np.sum(np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lq)))
        if 0 <= tokens[i] < vocab:
            logp[i] = lq[tokens[i]]
        key = np.where(np.isnan(z[i]), -np.inf, z[i])
        ids[i] = np.lexsort((np.arange(vocab), -key))[:top]
        lps[i] = lq[ids[i]]
    return logp, entropy, ids, lps


def teacher_distribution(ids, t, temperature: float, vocab: int) -> np.ndarray:
    """p over the whole vocabulary from one row's list (zeros without entries)."""
    out = np.zeros(vocab)
    valid = (ids >= 0) & (ids < vocab)
    if not valid.any():
        return out
    p = np.exp(log_softmax(t[valid] / temperature))
    np.add.at(out, ids[valid], p)
    return out


def distill(z, ids, t, labels, temperature: float, w: float, dloss):
    """Loss [rows] and gradient [rows, vocab] of distillation (labels may be None
    with w = 1)."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    for i in range(rows):
        if np.isneginf(z[i]).all():
            continue
        if w > 0:
            valid = (ids[i] >= 0) & (ids[i] < vocab)
            lq = log_softmax(z[i] / temperature)
            tv = np.asarray(t[i], np.float64)[valid] / temperature
            lp = log_softmax(tv) if valid.any() else tv
            terms = [np.exp(a) * (a - lq[j]) for a, j in zip(lp, ids[i][valid]) if not np.exp(a) == 0]
            loss[i] += w * temperature ** 2 * (np.sum(terms) if terms else 0.0)
            P = teacher_distribution(ids[i], np.asarray(t[i], np.float64), temperature, vocab)
            grad[i] += w * temperature * (np.exp(lq) * P.sum() - P)
        if w < 1 and 0 <= labels[i] < vocab:
            lh = log_softmax(z[i])
            loss[i] -= (1 - w) * lh[labels[i]]
            h = np.exp(lh)
            h[labels[i]] -= 1.0
            grad[i] += (1 - w) * h
        grad[i] *= dloss[i]
    return loss, grad
