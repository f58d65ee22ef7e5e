"""The operators on logits at the ends of their temperatures, and losses whose
terms pass fp32's range before their product with the temperature does not,
against the float64 definition.

Tolerances.  A teacher's probability and a softmax are held to 5e-5 of their size
(see test_gpu_logits.py), ln S to 2e-5.  The soft term is w T (T (sum p ln p + ln S)
- sum p d), d = z - max z: with |sum p ln p| and |ln S| at least 1 here or their
terms far below the others, it is off by at most 1e-4 of w T (T (1 + |sum p ln p| +
|ln S|) + sum p |d|), the hard one by 1e-4 (1 + its size)."""
import numpy as np
import pytest

import test_gpu_logits as base
from oracle import output_ops as ops

pytestmark = pytest.mark.gpu

LOWEST = {"bf16": -3.3895313892515355e38, "f32": -3.4028234663852886e38}


def soft_size(z, ids, t, T, w):
    out = np.zeros(len(z))
    for i in range(len(z)):
        p = ops.teacher_distribution(ids[i], t[i].astype(np.float64), T, z.shape[1])
        d = z[i] - z[i].max()
        on = p > 0
        lns = np.log(np.exp(d / T).sum())
        out[i] = w * T * (T * (1 + abs((p[on] * np.log(p[on])).sum()) + abs(lns)) + (p[on] * np.abs(d[on])).sum())
    return out


def check(z, ids, t, labels, dl, T, w, dtype):
    loss, grad = ops.distill(z, ids, t.astype(np.float64), labels, T, w, dl.astype(np.float64))
    hard = ops.distill(z, ids, t.astype(np.float64), labels, T, 0.0, dl.astype(np.float64))[0]
    d = base.on_device(z, dtype)
    for got, g in base.run_distill(d, ids, t, labels, dl, T, w, dtype, 0, 0):
        with np.errstate(over="ignore"):
            past = np.isinf(loss.astype(np.float32))
        tol = 1e-4 * (soft_size(z, ids, t, T, w) + (1 - w) * (1 + hard))
        assert (np.isinf(got) == past).all(), (got, loss)
        assert (np.abs(got - loss)[~past] <= tol[~past]).all(), (T, w, got, loss, tol)
        for i in range(len(z)):
            q = np.exp(ops.log_softmax(z[i] / T))
            h = np.exp(ops.log_softmax(z[i]))
            p = ops.teacher_distribution(ids[i], t[i].astype(np.float64), T, z.shape[1])
            one = np.arange(z.shape[1]) == labels[i]
            part = dl[i] * (w * T * (q + p) + (1 - w) * (h + one))
            tol_g = 1e-4 * part + (2.0 ** -8 * np.abs(grad[i]) if dtype == "bf16" else 0.0) + 1e-38
            assert (np.abs(g[i] - grad[i]) <= tol_g).all(), (T, w, i)


@pytest.mark.parametrize("dtype", base.DTYPES)
@pytest.mark.parametrize("vocab", [40, 5001, 70001, 140001])
@pytest.mark.parametrize("T", [2.0 ** -63, 1e-10, 0.01, 100.0, 1e10, 2.0 ** 63])
def test_distillation_at_the_ends(vocab, dtype, T):
    print(f"distill {vocab} {dtype} {T}", flush=True)
    rng = np.random.default_rng(vocab)
    z = base.as_stored(rng.normal(size=(6, vocab)) * 2.5, dtype)
    ids, t, labels, dl = base.lists_of(z, 6, 11)
    check(z, ids, t, labels, dl, T, 0.5, dtype)


@pytest.mark.parametrize("dtype", base.DTYPES)
@pytest.mark.parametrize("vocab", [40, 5001, 140001])
@pytest.mark.parametrize("T", [1e-10, 0.25, 0.7, 1.0])
def test_loss_of_a_listed_column_at_the_lowest_value(vocab, dtype, T):
    """d / T passes fp32's range, w T sum p d does not."""
    rng = np.random.default_rng(vocab)
    z = base.as_stored(rng.normal(size=(5, vocab)) * 2.5, dtype)
    ids, t, labels, dl = base.lists_of(z, 6, 12)
    ids[3, 0], ids[4] = ids[0, 0], ids[0]
    for i in range(5):
        z[i, ids[i, 0]] = LOWEST[dtype]
        labels[i] = ids[i, 1] if ids[i, 1] >= 0 and ids[i, 1] != ids[i, 0] else -1
    t[:, 0] = t.max(1)
    check(z, ids, t, labels, dl, T, 0.5, dtype)


@pytest.mark.parametrize("dtype", base.DTYPES)
@pytest.mark.parametrize("vocab", [9, 5000, 150001])
@pytest.mark.parametrize("T", [2.0 ** -126, 1e-10, 1e10, 3.4e38])
def test_scores_at_the_ends(vocab, dtype, T):
    z, tokens = base.rows_of(vocab, vocab)
    z = base.as_stored(z, dtype)
    T = float(np.float32(T))
    for top in (0, min(vocab, 20)):
        base.check_scores(z, tokens, top, T, base.score(base.on_device(z, dtype), tokens, top, T))
