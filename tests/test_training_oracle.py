"""Pins of the oracle of head, losses and checkpoints: gradients against central differences, known values, and the
properties that the formulas promise."""
import numpy as np
import pytest

from oracle import training_oracle as T


def differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        lo, hi = x.copy(), x.copy()
        lo[i] -= step
        hi[i] += step
        g[i] = (f(hi) - f(lo)) / (2 * step)
    return g


# central differences: step^2 / 6 times a third derivative of order one, and 1e-16 / step of cancellation
FD = 1e-8


@pytest.mark.parametrize("scale", [1.0, 0.5, -1.3])
def test_head_gradient_is_the_difference_quotient(scale):
    rng = np.random.default_rng(1)
    b, d, v = 5, 4, 7
    U, W, c = rng.standard_normal((b, d)), rng.standard_normal((v, d)), rng.standard_normal(b)
    labels = [0, 6, -1, 3, 7]      # two of them are not in the vocabulary
    dU, dW = T.head_bwd(U, W, labels, c, scale)
    assert np.abs(dU - differences(lambda u: c @ T.head_fwd(u, W, labels, scale)[0], U)).max() < FD
    assert np.abs(dW - differences(lambda w: c @ T.head_fwd(U, w, labels, scale)[0], W)).max() < FD
    assert not dU[2].any() and not dU[4].any()


def test_head_of_one_word_is_certain():
    logp, lse = T.head_fwd(np.ones((2, 3)), np.ones((1, 3)), [0, 5])
    assert logp.tolist() == [0.0, 0.0] and lse.tolist() == [3.0, 3.0]


@pytest.mark.parametrize("mean,smooth,margin", [(False, 0.0, 0.0), (True, 0.1, 0.5), (False, 1.0, -2.0)])
def test_preference_gradient_is_the_difference_quotient(mean, smooth, margin):
    rng = np.random.default_rng(2)
    off = [1, 4, 4, 9, 12, 13, 17]      # an empty sequence, a token before and two behind
    n = 19
    lp, ref = -rng.random(n) * 3, -rng.random(n) * 3
    mask = rng.integers(0, 2, n)
    args = (ref, mask, off, 0.7, smooth, margin, mean)
    g = T.preference(lp, *args)["dlogp"]
    assert np.abs(g - differences(lambda x: T.preference(x, *args)["loss"], lp)).max() < FD
    assert T.preference(lp, *args, grad_scale=3.0)["dlogp"] == pytest.approx(3 * g)


def test_preference_of_equal_answers():
    out = T.preference(np.zeros(4), None, None, [0, 2, 4], 0.3)
    assert out["loss"] == pytest.approx(np.log(2)) and out["dlogp"].tolist() == [-0.15, -0.15, 0.15, 0.15]


@pytest.mark.parametrize("by_sequence", [False, True])
@pytest.mark.parametrize("per_token", [False, True])
def test_policy_gradient_is_the_difference_quotient(by_sequence, per_token):
    rng = np.random.default_rng(3)
    off = [0, 3, 3, 8, 14]
    n = 16
    lp = -rng.random(n) * 2
    old, ref = lp + 0.4 * rng.standard_normal(n), lp + 0.3 * rng.standard_normal(n)
    mask = np.array([1] * 8 + [0] * 2 + [1] * 6)
    args = (old, ref, rng.standard_normal(n if per_token else 4), mask, off, 0.2, 0.28, 0.1, by_sequence, per_token)
    out = T.policy(lp, *args)
    assert 0 < out["clipped"] < 1
    assert np.abs(out["dlogp"] - differences(lambda x: T.policy(x, *args)["loss"], lp, 1e-6)).max() < FD


def test_policy_without_counted_tokens():
    out = T.policy(np.zeros(3), np.zeros(3), None, np.ones(1), np.zeros(3), [0, 3], 0.2, 0.2)
    assert out["loss"] == 0 and not out["dlogp"].any()


def test_checkpoints_are_within_half_a_step_and_repeat():
    rng = np.random.default_rng(4)
    X = (rng.standard_normal((40, 97)) * 10.0 ** rng.integers(-6, 6, (40, 1))).astype(np.float32)
    X = (X.view(np.uint32) & 0xFFFF0000).view(np.float32)      # bf16 numbers
    q, e = T.ckpt_pack(X)
    Y = T.ckpt_unpack(q, e, 97)
    step = np.repeat(2.0 ** (e.astype(np.float64) - 127), 32, axis=1)[:, :97]
    assert (np.abs(X.astype(np.float64) - Y) <= step / 2).all()
    assert np.abs(q).max(axis=1).min() >= 64      # the largest value of a group uses all seven bits
    q2, e2 = T.ckpt_pack(Y)
    assert (q2 == q).all() and (e2 == e).all()
    assert ((Y.view(np.uint32) & 0xFFFF) == 0).all()      # exact in bf16
