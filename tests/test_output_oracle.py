"""Pins of the float64 definitions of the operators around the layer's output
(oracle/output_ops.py): hand-worked values, other routes to the same result and
finite differences, and planted mistakes that the pins have to find."""
import math

import numpy as np
import pytest

from oracle import output_ops as ops


def bits(x):
    """float -> bf16 pattern (values here are exact in bf16)."""
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


# ---- microscaled 4 bits -------------------------------------------------------
def check_nearest(nearest):
    ties = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}       # to the even code
    for y, code in ties.items():
        assert nearest(np.array([y]))[0] == code and nearest(np.array([-y]))[0] == code + 8, y
        eps = 1e-9
        assert nearest(np.array([y - eps]))[0] == (code if code % 2 == 0 and ops.E2M1[code] < y else code - 1), y
        assert nearest(np.array([y + eps]))[0] == (code if ops.E2M1[code] > y else code + 1), y
    for code, v in enumerate(ops.E2M1):
        assert nearest(np.array([v]))[0] == code
    assert nearest(np.array([7.9]))[0] == 7 and nearest(np.array([-100.0]))[0] == 15
    assert nearest(np.array([-0.0]))[0] == 8


def test_nearest_code():
    check_nearest(ops.mx4_nearest)


@pytest.mark.parametrize("wrong", [
    lambda y: np.argmin(np.abs(np.abs(y)[..., None] - ops.E2M1), -1) + 8 * np.signbit(y),      # ties down
    lambda y: 7 - np.argmin(np.abs(np.abs(y)[..., None] - ops.E2M1[::-1]), -1) + 8 * np.signbit(y),   # ties up
    lambda y: ops.mx4_nearest(np.abs(y)),                                                     # no sign
    lambda y: ops.mx4_nearest(y / 2)])
def test_planted_rounding_mistakes_are_found(wrong):
    with pytest.raises(AssertionError):
        check_nearest(wrong)


def test_block_scale_by_hand():
    x = np.zeros((1, 64))
    x[0, :3] = [6.0, -3.0, 0.7]          # exponent of 6 is 2: scale 2^0
    x[0, 32:34] = [0.1, 1.99]            # exponent of 1.99 is 0: scale 2^-2, 1.99 -> 7.96 -> 6
    codes, scales = ops.mx4_encode(bits(x))
    q = ops.mx4_decode(codes, scales, 64)[0]
    assert scales[ops.mx4_scale_place(0, 0, 1)] == 127 and scales[ops.mx4_scale_place(0, 1, 1)] == 125
    assert list(q[:3]) == [6.0, -3.0, 0.5] and list(q[32:34]) == [0.125, 1.5]
    assert codes[0, 0] == 7 + 16 * 13 and codes[0, 1] == 1
    assert not codes[0, 32:].any() and codes.shape == (1, 128)


def test_representable_values_survive_and_extremes():
    rng = np.random.default_rng(3)
    code = rng.integers(0, 16, (5, 96))
    code[:, ::32] = 7                                             # every block reaches 6
    x = np.where(code < 8, 1, -1) * ops.E2M1[code % 8] * 2.0 ** rng.integers(-20, 20, (5, 3)).repeat(32, 1)
    codes, scales = ops.mx4_encode(bits(x))
    assert np.array_equal(ops.mx4_decode(codes, scales, 96), x)
    tiny = np.full((1, 32), 2.0 ** -133)                          # below the smallest scale's half step
    assert ops.mx4_encode(bits(tiny))[1].max() == 0 and not ops.mx4_decode(*ops.mx4_encode(bits(tiny)), 32).any()
    bad = np.zeros((2, 64))
    bad[0, 5], bad[1, 40] = np.inf, np.nan
    q = ops.mx4_decode(*ops.mx4_encode(bits(bad)), 64)
    assert np.isnan(q[0, :32]).all() and not q[0, 32:].any() and not q[1, :32].any() and np.isnan(q[1, 32:]).all()


def test_scale_places_are_a_bijection():
    for rows, blocks in ((1, 8), (64, 8), (65, 16), (200, 24)):
        at = {int(ops.mx4_scale_place(i, b, -(-rows // 64) * 64)) for i in range(-(-rows // 64) * 64) for b in range(blocks)}
        assert at == set(range(-(-rows // 64) * (blocks // 8) * 512))


def test_linear_is_the_product_of_the_decoded_matrices():
    rng = np.random.default_rng(4)
    x, w = (bits(rng.integers(-3, 4, s).astype(float)) for s in ((3, 40), (5, 40)))
    xq, wq = ops.mx4_decode(*ops.mx4_encode(x), 40), ops.mx4_decode(*ops.mx4_encode(w), 40)
    y = ops.mx4_linear(x, *ops.mx4_encode(w))
    for i in range(3):
        for j in range(5):
            assert y[i, j] == sum(xq[i, l] * wq[j, l] for l in range(40))


# ---- rows of logits -----------------------------------------------------------
def test_uniform_and_two_point_rows():
    z = np.zeros((1, 8))
    logp, entropy, ids, lps = ops.token_logprobs(z, [3], 0.5, 3)
    assert math.isclose(logp[0], -math.log(8)) and math.isclose(entropy[0], math.log(8))
    assert list(ids[0]) == [0, 1, 2] and np.allclose(lps, -math.log(8))
    z = np.array([[0.0, math.log(3.0)]])
    logp, entropy, ids, _ = ops.token_logprobs(z, [0], 1.0, 2)
    assert math.isclose(logp[0], math.log(0.25))
    assert math.isclose(entropy[0], 0.25 * math.log(4) + 0.75 * math.log(4 / 3)) and list(ids[0]) == [1, 0]


def test_special_rows():
    inf, nan = np.inf, np.nan
    z = np.array([[-inf, -inf, -inf], [1.0, nan, 3.0], [0.0, inf, 0.0], [1.0, -inf, 1.0], [0.0, -0.0, -1.0]])
    logp, entropy, ids, lps = ops.token_logprobs(z, [0, 0, 0, 1, -1], 1.0, 2)
    assert logp[0] == -inf and entropy[0] == 0 and list(ids[0]) == [0, 1] and np.isneginf(lps[0]).all()
    assert np.isnan(logp[1:3]).all() and np.isnan(entropy[1:3]).all() and np.isnan(lps[1:3]).all()
    assert list(ids[1]) == [2, 0] and list(ids[2]) == [1, 0]
    assert logp[3] == -inf and math.isclose(entropy[3], math.log(2)) and list(ids[3]) == [0, 2]
    assert logp[4] == 0 and list(ids[4]) == [0, 1]


def _case(seed=0, rows=4, vocab=11, top=5):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(rows, vocab)) * 2
    ids = np.stack([rng.permutation(vocab)[:top] for _ in range(rows)])
    ids[0, 3:] = -1                      # a shorter list
    ids[1, 4] = ids[1, 0]                # one id twice
    ids[2, :] = -1                       # none
    t = rng.normal(size=(rows, top)) * 2
    labels = rng.integers(0, vocab, rows)
    labels[3] = -100
    labels[1] = ids[1, 0]
    return z, ids, t, labels, rng.uniform(0.5, 1.5, rows)


def check_gradient(distill):
    for T, w in ((1.0, 1.0), (2.0, 0.5), (0.7, 0.25), (1.0, 0.0)):
        z, ids, t, labels, dl = _case()
        loss, grad = distill(z, ids, t, labels, T, w, dl)
        h = 1e-5
        for j in range(z.shape[1]):
            zp, zm = z.copy(), z.copy()
            zp[:, j] += h
            zm[:, j] -= h
            num = (distill(zp, ids, t, labels, T, w, dl)[0] - distill(zm, ids, t, labels, T, w, dl)[0]) / (2 * h) * dl
            assert np.abs(num - grad[:, j]).max() < 1e-8, (T, w, j)
        # adding a number to a row of logits, the student's or the teacher's, changes nothing
        shifted = distill(z + 3.0, ids, t - 5.0, labels, T, w, dl)
        assert np.allclose(shifted[0], loss) and np.allclose(shifted[1], grad) and np.abs(grad.sum(1)).max() < 1e-12
    # the soft loss is 0 where the student's softmax is the teacher's
    z, ids, t, labels, dl = _case()
    full = np.arange(z.shape[1])[None].repeat(len(z), 0)
    loss, grad = distill(z, full, z, None, 2.0, 1.0, dl)
    assert np.abs(loss).max() < 1e-12 and np.abs(grad).max() < 1e-12
    # and the cross entropy of the label at w = 0
    loss, _ = distill(z, ids, t, labels, 2.0, 0.0, dl)
    assert np.allclose(loss, [-(z[i] - np.log(np.exp(z[i]).sum()))[l] if l >= 0 else 0.0 for i, l in enumerate(labels)])


def test_distillation_gradient_is_the_loss_difference():
    check_gradient(ops.distill)


@pytest.mark.parametrize("name", ["T", "1/T", "sign", "label", "mass"])
def test_planted_gradient_mistakes_are_found(name):
    def wrong(z, ids, t, labels, T, w, dl):
        loss, grad = ops.distill(z, ids, t, labels, T, w, dl)
        soft = ops.distill(z, ids, t, None, T, 1.0, dl)[1] * w
        if name == "T":
            grad = grad + soft * (T - 1)
        elif name == "1/T":
            grad = grad + soft * (1 / T - 1)
        elif name == "sign":
            grad = -grad
        elif name == "label":
            grad = np.where(np.arange(z.shape[1]) == (labels if labels is not None else ids[:, 0])[:, None], 0.0, grad)
        elif name == "mass":       # an empty list as if it had mass
            grad = grad + w * T * dl[:, None] * np.exp(z - z.max(1, keepdims=True)) * (ids < 0).all(1)[:, None]
        return loss, grad
    with pytest.raises(AssertionError):
        check_gradient(wrong)
