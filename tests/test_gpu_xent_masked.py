"""Cross entropy without logits where a leading part of the vocabulary is masked: its
logits are minus infinity or the type's lowest value, and all others lie far below zero.
The reference of the powers then has to move down in a later piece than the first.
Expected: the definition over the columns that are left, with test_gpu_xent's bounds."""
import numpy as np
import pytest

from test_gpu_xent import bounds, case, close, f64, run, to_bits

pytestmark = pytest.mark.gpu


def masked(rows, vocab, k, leading, fill, level):
    """Columns below `leading` masked by `fill` in W's column 0, all logits shifted by `level`."""
    x, w, labels, d = case(rows, vocab, k, rows + leading, spread=1.0, sure=1.0)
    x, w = f64(x), f64(w)
    x[:, 0], w[:, 0] = 1.0, 0.0
    x[:, 1], w[:, 1] = level, 1.0
    known = (labels >= 0) & (labels < vocab)
    labels = np.where(known, leading + labels % (vocab - leading), labels).astype(np.int32)
    x, w = to_bits(x), to_bits(w)
    w[:leading, 0] = fill
    return x, w, labels, d


def expected(x, w, labels, d, leading):
    at = np.where((labels >= leading) & (labels < len(w)), labels - leading, -1)
    return bounds(f64(x), f64(w[leading:]), at, d.astype(np.float64))


# three pieces of 7680 columns or so, joined or carried by 128 x 256 tiles; few rows, one piece
@pytest.mark.parametrize("rows,vocab,k,leading", [(4100, 20011, 72, 9000), (4100, 20011, 72, 17000), (40, 6000, 72, 3000)])
@pytest.mark.parametrize("fill", [0xFF80, 0xFF7F])
@pytest.mark.parametrize("level", [-300.0, -96.0, -20.0])
def test_masked_first_part(rows, vocab, k, leading, fill, level):
    print(f"xent masked {rows} x {vocab} x {k}, {leading} at {fill:#x}, others near {level}", flush=True)
    x, w, labels, d = masked(rows, vocab, k, leading, fill, level)
    (loss, dX, dW), (t_loss, t_dX, t_dW) = expected(x, w, labels, d, leading)
    for how, dw in (("step", False), ("step", True), ("two", True)):
        got = run(x, w, labels, d, how, True, dw)
        assert np.isfinite(got[0]).all(), how
        assert (np.abs(got[0] - loss) <= t_loss * (1 + 1e-6)).all(), how
        # (column 0 of dX is 0 times the mask)
        assert (np.abs(got[1] - dX)[:, 1:] <= t_dX[:, 1:] * (1 + 1e-6)).all(), how
        if dw:
            assert (got[2][:leading] == 0).all() and (np.abs(got[2][leading:] - dW) <= t_dW * (1 + 1e-6)).all(), how


def test_masked_first_part_beside_rows_that_are_not():
    """Rows masked and rows not in the same tiles: each keeps a reference of its own."""
    rows, vocab, k, leading = 4100, 20011, 72, 9000
    x, w, labels, d = masked(rows, vocab, k, leading, 0xFF7F, -300.0)
    free = np.arange(rows) % 3 == 0
    x[free, 0] = 0                                             # 0 x the lowest value: not masked
    x[np.arange(rows) % 6 == 0, 1] = to_bits(np.array([5.0]))[0]
    (want, tol) = expected(x[~free], w, labels[~free], d[~free], leading)
    plain = w.copy()
    plain[:, 0] = 0
    (want_f, tol_f) = bounds(f64(x[free]), f64(plain), labels[free], d[free].astype(np.float64))
    for how in ("step", "two"):
        loss, dX, _ = run(x, w, labels, d, how)
        close((loss[~free], dX[~free][:, 1:], None), (want[0], want[1][:, 1:], None), (tol[0], tol[1][:, 1:], None), how)
        close((loss[free], dX[free][:, 1:], None), (want_f[0], want_f[1][:, 1:], None), (tol_f[0], tol_f[1][:, 1:], None), how)


@pytest.mark.parametrize("rows,vocab,k", [(1, 300, 8), (40, 6000, 72), (300, 1500, 64), (4100, 20011, 72)])
@pytest.mark.parametrize("fill", [0xFF80, 0xFF7F, 0xE2AD, 0xD015])
@pytest.mark.parametrize("level", [-300.0, 0.0, 300.0])
def test_the_label_alone_is_left(rows, vocab, k, fill, level):
    """Every column but the label's masked, by minus infinity, the lowest value, -1.6e21 or
    -1e10: probability 1, so that loss and gradients are 0."""
    print(f"xent label alone {rows} x {vocab} x {k}, mask {fill:#x}, near {level}", flush=True)
    x, w, labels, d = masked(rows, vocab, k, vocab - 1, fill, level)
    known = (labels >= 0) & (labels < vocab)
    assert (labels[known] == vocab - 1).all()
    for how, dw in (("step", False), ("step", True), ("two", True)):
        loss, dX, dW = run(x, w, labels, d, how, True, dw)
        assert (loss == 0).all() and (dX[:, 1:] == 0).all(), how
        assert not dw or (dW == 0).all(), how
