"""Cross entropy without logits on finite logits of any size: masks by large negative
numbers, and rows whose logits are large.

Masked columns count as probability 0 (their difference from the row's largest logit
passes 1e9): the definition over the columns that are left, with test_gpu_xent's bounds.

Large logits are whole multiples of their own spacing, formed from two exact products, so
that fp32 holds them and their differences exactly; the definition then knows no rounding
but the kernels' own.  The difference D to the largest logit is exact, its product with
log2 e off by 2^-22 of at most 1.45 D: with D <= 7.5 a power is off by 11 2^-22 of itself at
most, and where D is larger, terms e^-D count by D e^-D < 3/8.  A sum of powers has 64 +
tiles roundings of 2^-24 (as in test_gpu_xent), so a loss is off by 2^-18 + (64 + tiles)
2^-24 and, being a number of the logits' size taken from fp64, 2^-23 of itself.  A row's
numbers for the two-call form are held in bf16 from |log sum| 2^16 on and off by half an
fp32 spacing of the logarithm, 2^-9, below; G is bf16: 2^-9 + 2^-9 + 2^-9 and the result's
2^-9, with the above below 2^-6 of sum |g||w|."""
import numpy as np
import pytest

from oracle import train_ops as ops
from test_gpu_xent import bounds, case, f64, run, to_bits

pytestmark = pytest.mark.gpu


def losses(z, labels):
    """The definition with the label's difference to the largest taken first: log T + 2^60 in
    fp64 would be 2^60."""
    d = z.max(axis=1) - z[np.arange(len(z)), np.maximum(labels, 0)]
    return np.where(labels >= 0, np.log(np.exp(z - z.max(axis=1, keepdims=True)).sum(axis=1)) + d, 0.0)


# one piece with tiles' own references; one piece; several pieces
@pytest.mark.parametrize("rows,vocab,k", [(40, 3000, 72), (300, 5000, 136), (1000, 15000, 264), (4100, 20011, 72)])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -6e29, -1e31, -3e38])
@pytest.mark.parametrize("where", ["first", "last"])
def test_finite_masks(rows, vocab, k, mask, where):
    print(f"xent mask {mask} {where} of {rows} x {vocab} x {k}", flush=True)
    x, w, labels, d = case(rows, vocab, k, rows, spread=1.0, sure=1.0)
    x, w = f64(x), f64(w)
    kept = np.arange(vocab // 2, vocab) if where == "first" else np.arange(0, vocab // 2)
    x[:, 0], w[:, 0] = 1.0, mask
    w[kept, 0] = 0.0
    known = (labels >= 0) & (labels < vocab)
    at = np.where(known, labels % len(kept), -1)
    labels = np.where(known, kept[at], labels).astype(np.int32)
    x, w = to_bits(x), to_bits(w)
    (loss, dX, dW), (t_loss, t_dX, t_dW) = bounds(f64(x), f64(w[kept]), at, d.astype(np.float64))
    for how, dw in (("step", False), ("step", True), ("two", True)):
        got = run(x, w, labels, d, how, True, dw)
        assert (np.abs(got[0] - loss) <= t_loss * (1 + 1e-6)).all(), how
        assert (np.abs(got[1] - dX) <= t_dX * (1 + 1e-6)).all(), how
        if dw:
            rest = np.ones(vocab, bool)
            rest[kept] = False
            assert (got[2][rest] == 0).all() and (np.abs(got[2][kept] - dW) <= t_dW * (1 + 1e-6)).all(), how


@pytest.mark.parametrize("rows,vocab,k", [(5, 700, 16), (40, 3000, 64), (300, 1500, 64), (1000, 15000, 64), (4100, 9001, 16)])
@pytest.mark.parametrize("power", [10, 15, 17, 20, 27, 29, 33, 60, 100, 125])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_large_logits(rows, vocab, k, power, sign):
    """z = sign 2^power - j u, j = 0 .. 15, u a spacing of such numbers or 1/2, whichever is more."""
    print(f"xent far {sign} 2^{power}, {rows} x {vocab} x {k}", flush=True)
    rng = np.random.default_rng(power + rows)
    unit = max(0.5, 2.0 ** (power - 16))
    j = rng.integers(0, 16, vocab)
    w = np.zeros((vocab, k))
    w[:, 0], w[:, 1] = 1.0, -j
    w[:, 2:] = rng.normal(size=(vocab, k - 2))
    x = np.zeros((rows, k))
    x[:, 0], x[:, 1] = sign * 2.0 ** power, unit
    x[::4, 0] = 1.0                                             # ordinary rows among them
    x[::4, 1] = 0.5
    labels = rng.integers(0, vocab, rows).astype(np.int32)
    labels[2::5] = -100
    d = rng.normal(size=rows).astype(np.float32)
    x, w = to_bits(x), to_bits(w)
    fx, fw, fd = f64(x), f64(w), d.astype(np.float64)
    _, g, dX, dW = ops.xent(fx, fw, labels, fd)
    loss = losses(fx @ fw.T, labels)
    for how, dw in (("step", False), ("step", True), ("two", True)):
        got = run(x, w, labels, d, how, True, dw)
        tol = 2.0 ** -18 + (64 + -(-vocab // 128)) * 2.0 ** -24 + 2.0 ** -23 * np.abs(loss)
        assert (np.abs(got[0] - loss) <= tol).all(), (how, np.max(np.abs(got[0] - loss) - tol))
        assert (np.abs(got[1] - dX) <= 2.0 ** -6 * (np.abs(g) @ np.abs(fw)) + 2.0 ** -120).all(), how
        if dw:
            assert (np.abs(got[2] - dW) <= 2.0 ** -6 * (np.abs(g).T @ np.abs(fx)) + 2.0 ** -120).all(), how


@pytest.mark.parametrize("rows", [7, 300])
def test_all_logits_at_one_value(rows):
    """A row masked as a whole by a finite number: every column alike, the loss log(vocab)."""
    vocab, k = 2000, 32
    rng = np.random.default_rng(0)
    w = np.zeros((vocab, k))
    w[:, 0], w[:, 1:] = 1.0, rng.normal(size=(vocab, k - 1))
    x = np.zeros((rows, k))
    x[:, 0] = rng.choice([-3e38, -1e31, -1e30, -7e29, -1e10, 1e10, 2.4e38, 3e38], rows)
    labels, d = rng.integers(0, vocab, rows).astype(np.int32), np.ones(rows, np.float32)
    x, w = to_bits(x), to_bits(w)
    _, g, dX, _ = ops.xent(f64(x), f64(w), labels, d.astype(np.float64))
    for how in ("step", "two"):
        loss, got, _ = run(x, w, labels, d, how)
        assert (np.abs(loss - np.log(vocab)) <= 2.0 ** -18 + 80 * 2.0 ** -24 + 2.0 ** -23 * np.log(vocab)).all(), how
        assert (np.abs(got - dX) <= 2.0 ** -6 * (np.abs(g) @ np.abs(f64(w)))).all(), how
