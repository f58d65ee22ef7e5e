"""Pins of the float64 definitions of the operators of a fine-tuning step
(oracle/train_ops.py): by hand, by another route, by differences, and planted
mistakes that the pins have to find."""
import numpy as np
import pytest

import oracle
from oracle import train_ops as ops


def bits(x):
    return oracle.f64_to_bf16_bits(np.asarray(x, np.float64))


# ---- 8 bits ----------------------------------------------------------------------
def nearest_by_search(v):
    """Every magnitude's distance, ties to the even code."""
    d = np.abs(np.abs(v) - ops.E4M3)
    best = np.flatnonzero(d == d.min())
    return int(best[best % 2 == 0][0] if len(best) > 1 else best[0]) + (128 if np.signbit(v) else 0)


def test_magnitudes():
    assert len(ops.E4M3) == 127 and ops.E4M3[0] == 0 and ops.E4M3[1] == 2.0 ** -9 and ops.E4M3[8] == 2.0 ** -6
    assert ops.E4M3[56] == 1.0 and ops.E4M3[126] == 448.0 and (np.diff(ops.E4M3) > 0).all()


def _values():
    mid = (ops.E4M3[1:] + ops.E4M3[:-1]) / 2
    return np.concatenate([ops.E4M3, -ops.E4M3, mid, -mid, mid * (1 - 1e-9), mid * (1 + 1e-9), [0.0, -0.0, 447.9, 1e-12]])


def test_nearest_code():
    v = _values()
    assert ops.fp8_nearest(v).tolist() == [nearest_by_search(x) for x in v]


@pytest.mark.parametrize("wrong", [lambda v: ops.fp8_nearest(v * (1 + 1e-7)), lambda v: ops.fp8_nearest(np.abs(v)),
                                   lambda v: ops.fp8_nearest(np.trunc(v * 512) / 512)])
def test_planted_rounding_mistakes_are_found(wrong):
    v = _values()
    assert wrong(v).tolist() != [nearest_by_search(x) for x in v]


def test_scale_by_hand():
    x = np.zeros((3, 264))
    x[0, 0], x[0, 130], x[1, 5], x[2, 263] = 448.0, 449.0, -896.0, 2.0 ** -133
    s = ops.fp8_scale_bytes(x, 1)
    assert s.tolist() == [[127, 128, 0], [128, 0, 0], [0, 0, 0]]
    assert ops.fp8_scale_bytes(x, 128).tolist() == [[128, 128, 0]]
    x[1, 6] = np.inf
    assert ops.fp8_scale_bytes(x, 1)[1, 0] == 255 and ops.fp8_scale_bytes(x, 128)[0, 0] == 255


@pytest.mark.parametrize("block_rows", [1, 128])
def test_encode_keeps_representable_values_and_is_within_half_a_step(block_rows):
    rng = np.random.default_rng(block_rows)
    x = ops._f64(bits(rng.normal(size=(200, 300)) * 2.0 ** rng.integers(-30, 30, (200, 1))))
    c, s = ops.fp8_encode(bits(x), block_rows)
    y = ops.fp8_decode(c, s, 300, block_rows)
    top = np.maximum.reduceat(np.abs(x), np.arange(0, 300, 128), axis=1)
    if block_rows == 128:
        top = np.stack([top[:128].max(0)] * 128 + [top[128:].max(0)] * 72)
    unit = np.repeat(top, 128, axis=1)[:, :300] / 448 * 2      # the scale is below twice the smallest that would do
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), unit * 2.0 ** -10)).all()
    assert c.shape == (200, 384) and (c[:, 300:] == 0).all()
    again = ops.fp8_encode(bits(y), block_rows)
    assert np.array_equal(ops.fp8_decode(*again, 300, block_rows), y)


def test_scale_places_are_a_bijection():
    i, b = np.indices((130, 3))
    assert len(set(ops.fp8_scale_place(i, b, 130).reshape(-1).tolist())) == 390
    assert ops.fp8_scale_place(0, 0, 130) == 0 and ops.fp8_scale_place(17, 1, 130) == 3 * 64 + 5
    assert ops.fp8_scale_place(64, 0, 130) == 64


# ---- cross entropy -----------------------------------------------------------------
def _case(seed=3, rows=7, vocab=11, k=8):
    rng = np.random.default_rng(seed)
    x, w = rng.normal(size=(rows, k)), rng.normal(size=(vocab, k))
    labels = rng.integers(0, vocab, rows)
    labels[1], labels[2] = -100, vocab
    return x, w, labels, rng.normal(size=rows)


def test_loss_by_hand_and_rows_without_a_label():
    x, w = np.array([[1.0, 0.0], [0.0, 2.0]]), np.array([[np.log(3.0), 0.0], [0.0, 0.0]])
    loss, g, dx, _ = ops.xent(x, w, np.array([1, 0]), np.array([1.0, 2.0]))
    assert np.allclose(loss, [np.log(4.0), np.log(2.0)]) and np.allclose(g, [[0.75, -0.75], [-1.0, 1.0]])
    assert np.allclose(dx[0], [0.75 * np.log(3.0), 0.0])
    x, w, labels, d = _case()
    loss, g, dx, dw = ops.xent(x, w, labels, d)
    assert (loss[1:3] == 0).all() and (g[1:3] == 0).all() and (dx[1:3] == 0).all()
    keep = np.array([0, 3, 4, 5, 6])
    assert np.allclose(ops.xent(x[keep], w, labels[keep], d[keep])[3], dw)


def _differences(fn):
    x, w, labels, d = _case()
    _, _, dx, dw = fn(x, w, labels, d)
    worst, h = 0.0, 1e-6
    for t, grad in ((x, dx), (w, dw)):
        for i in range(t.shape[0]):
            for j in range(t.shape[1]):
                old = t[i, j]
                t[i, j] = old + h
                up = (ops.xent(x, w, labels, d)[0] * d).sum()
                t[i, j] = old - h
                down = (ops.xent(x, w, labels, d)[0] * d).sum()
                t[i, j] = old
                worst = max(worst, abs((up - down) / (2 * h) - grad[i, j]))
    return worst


def test_gradients_are_the_losses_differences():
    # a central difference is off by h^2 / 6 of a third derivative (order 10) and 2^-53 / h of the loss (order 10)
    assert _differences(ops.xent) < 1e-7


@pytest.mark.parametrize("wrong", ["no label", "unscaled", "transposed sign", "labels shifted"])
def test_planted_gradient_mistakes_are_found(wrong):
    def mistaken(x, w, labels, d):
        loss, g, dx, dw = ops.xent(x, w, labels, d)
        if wrong == "no label":
            g = np.maximum(g / np.where(d == 0, 1, d)[:, None], 0) * d[:, None]
        elif wrong == "unscaled":
            g = g / d[:, None]
        elif wrong == "transposed sign":
            return loss, g, dx, -dw
        else:
            return ops.xent(x, w, labels + 1, d)
        return loss, g, g @ w, g.T @ x
    assert _differences(mistaken) > 1e-3


def test_a_sure_row_keeps_its_digits():
    x, w = np.array([[1.0, 0.0]]), np.array([[50.0, 0.0], [0.0, 0.0], [0.0, 1.0]])
    loss, g, _, _ = ops.xent(x, w, np.array([0]), np.array([1.0]))
    assert np.isclose(loss[0], 2 * np.exp(-50), rtol=1e-12) and np.isclose(-g[0, 0], 2 * np.exp(-50), rtol=1e-12)


# ---- dropout -----------------------------------------------------------------------
@pytest.mark.parametrize("seed,offset", [(0, 0), (2 ** 64 - 3, 7), (99, 2 ** 64 - 1)])
def test_draws_are_the_keep_masks_and_numpys(seed, offset):
    m, k, p = 3, 24, 0.3
    mask = oracle.dropout_keep_philox(seed, offset, p, m, k)
    kept = ops.dropout_kept(seed, offset, p, (m, k))
    assert np.array_equal(np.unpackbits(mask, axis=1, bitorder="little").astype(bool), kept)
    ctr = (int(offset) - 1) % 2 ** 256                        # numpy's generator advances before it draws
    words64 = [np.array(v, np.uint64) for v in ([(ctr >> (64 * i)) & (2 ** 64 - 1) for i in range(4)], [seed, 0])]
    gen = np.random.Philox(counter=words64[0], key=words64[1])
    words = np.asarray(gen.random_raw(12), np.uint64).astype("<u8").view("<u2")
    assert np.array_equal(words[:40], ops.dropout_draws(seed, offset, 40))


def test_rates():
    assert ops.dropout_kept(1, 0, 0.0, (4, 100)).all()
    kept = ops.dropout_kept(1, 0, 0.3, (8000,)).mean()
    assert abs(kept - 0.7) < 5 * (0.21 / 8000) ** 0.5
    assert not (ops.dropout_kept(1, 0, 0.5, (400,)) & ~ops.dropout_kept(1, 0, 0.3, (400,))).any()
