"""The policy loss where an exponential of a difference of log-probabilities is beyond fp32 and the result is not."""
import numpy as np
import pytest

from oracle import training_oracle as T
from tests.test_gpu_loss import ONCE, f32, offsets, run_policy

pytestmark = pytest.mark.gpu
TOL = 16 * 2.0 ** -24      # of the size of a token's terms: see check_policy of the loss tests

SIZES = [(3, 5), (16, 20), (1, 700), (40, 60), (3, 3000)]      # one workgroup, and slices


def far_apart(rng, n, at, share=0.2):
    """fp32 log-probabilities of n tokens and others that are `at` above or below them for some tokens, near them for the rest."""
    lp = (-3 * rng.random(n)).astype(np.float32)
    d = 0.2 * rng.standard_normal(n)
    far = rng.random(n) < share
    far[0] = True
    d[far] = rng.choice(np.asarray(at, np.float64), int(far.sum()))
    return lp, (lp - d).astype(np.float32), far


def check(got, want, loss_size):
    assert (np.abs(got["dlogp"] - want["dlogp"]) <= TOL * want["size"]).all()
    assert abs(got["loss"][0] - want["loss"]) <= TOL * loss_size
    assert abs(got["kl"][0] - want["kl"]) <= TOL * (1 + 100) * want["kl"]      # exp(q) of a |q| of 100 that is rounded to fp32
    assert abs(got["clipped"][0] - want["clipped"]) <= ONCE


@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("by_seq", [False, True])
@pytest.mark.parametrize("seqs,mean_len", SIZES)
def test_a_ratio_beyond_fp32_without_an_advantage(seqs, mean_len, by_seq, per_token):
    """Answers that all have the same reward: an advantage of zero, at any distance from the old policy."""
    rng = np.random.default_rng([seqs, mean_len, int(by_seq), int(per_token)])
    off = offsets(rng, seqs, mean_len, empty=0.0)
    off[1:] += 1
    n = int(off[-1])
    lp, old, far = far_apart(rng, n, [88.8, 100, 700, -100, -700])
    if per_token:
        adv = np.where(far, 0.0, rng.standard_normal(n)).astype(np.float32)
        size = 3.0 * np.abs(adv).max()
    else:
        adv, size = np.zeros(seqs, np.float32), 0.0
    got = run_policy(lp, old, None, adv, None, off, by_seq=by_seq, per_token=per_token)
    want = T.policy(lp, old, None, adv, None, off, f32(0.2), f32(0.28), 0.0, by_seq, per_token)
    check(got, want, size)
    if not per_token:
        assert got["loss"][0] == 0 and not got["dlogp"].any()


@pytest.mark.parametrize("by_seq", [False, True])
@pytest.mark.parametrize("seqs,mean_len", SIZES)
def test_a_kl_that_is_only_watched(seqs, mean_len, by_seq):
    """kl_coef = 0 and a reference: its distance is reported, and no part of the loss or the gradient."""
    rng = np.random.default_rng([seqs, mean_len, int(by_seq), 2])
    off = offsets(rng, seqs, mean_len, empty=0.0)
    off[1:] += 1
    n = int(off[-1])
    lp, ref, _ = far_apart(rng, n, [-88.8, -90, 100, 300], 0.02)      # exp(90) times 1 / n is an fp32 number
    old = (lp + 0.2 * rng.standard_normal(n)).astype(np.float32)
    adv = rng.standard_normal(seqs).astype(np.float32)
    got = run_policy(lp, old, ref, adv, None, off, kl=0.0, by_seq=by_seq)
    want = T.policy(lp, old, ref, adv, None, off, f32(0.2), f32(0.28), 0.0, by_seq, False)
    assert want["kl"] > 1e30 or n < 20
    if want["kl"] < 3e38:
        check(got, want, 3.0 * np.abs(adv).max())
    without = run_policy(lp, old, None, adv, None, off, kl=0.0, by_seq=by_seq)
    assert np.array_equal(without["dlogp"], got["dlogp"])
    # the same terms, added up in another order: below 1e4 * 2^-53 of their size in fp64, then a unit of fp32
    assert abs(without["loss"][0] - got["loss"][0]) <= ONCE * abs(got["loss"][0]) + 1e4 * 2.0 ** -53 * 3.0 * np.abs(adv).max()


def test_the_lowest_values_of_the_type():
    low = np.finfo(np.float32).min
    lp = np.array([-1, low, -1, -2, low, -1, -3], np.float32)
    old = np.array([low, -1, -1, low, low, -2, -3], np.float32)
    ref = np.array([-1, -2, low, -1, -1, -2, -3], np.float32)      # token 4: ref - logp is 3.4e38
    got = run_policy(lp, old, ref, np.zeros(1, np.float32), None, np.array([0, 7], np.int64), kl=0.0)
    assert got["loss"][0] == 0 and not got["dlogp"].any() and got["clipped"][0] == 0 and got["kl"][0] == np.inf


def test_what_is_not_a_number_stays_one():
    lp = np.array([np.nan, -1, -2], np.float32)
    got = run_policy(lp, np.full(3, -1, np.float32), None, np.zeros(1, np.float32), None, np.array([0, 3], np.int64))
    assert np.isnan(got["loss"][0]) and np.isnan(got["dlogp"]).tolist() == [True, False, False]


@pytest.mark.parametrize("by_seq", [False, True])
@pytest.mark.parametrize("seqs,mean_len", [(16, 30), (1, 700), (40, 600), (3, 30000)])
def test_a_gradient_that_its_weight_brings_back_into_fp32(seqs, mean_len, by_seq):
    """rho A, the KL term and grad_scale times either beyond 3.4e38, their share of the batch below it."""
    rng = np.random.default_rng([seqs, mean_len, int(by_seq), 3])
    off = (1 + np.arange(seqs + 1) * mean_len).astype(np.int64)
    n, every = int(off[-1]) + 2, seqs * mean_len
    top = np.log(3.4e38) + 0.8 * np.log(every)      # exp() of it times 1 / every: an fp32 number
    lp = (-3 * rng.random(n)).astype(np.float32)
    near = lambda s: (lp + s * rng.standard_normal(n)).astype(np.float32)      # noqa: E731
    adv = -1 - rng.random(n).astype(np.float32)      # not clipped from above
    for what, scale in (("ratio", 1.0), ("kl", 1.0), ("scale", 1e37)):
        old, ref = near(0.2), near(0.2)
        at = 1 + int(rng.integers(0, every - 5))
        if what == "ratio":
            old[at:at + 5] = lp[at:at + 5] - np.float32(top - 1)
        elif what == "kl":
            ref[at:at + 5] = lp[at:at + 5] + np.float32(top)
        else:
            adv[at:at + 5] *= 60
        got = run_policy(lp, old, ref, adv, None, off, kl=0.05, by_seq=by_seq, per_token=True, grad_scale=scale)
        want = T.policy(lp, old, ref, adv, None, off, f32(0.2), f32(0.28), f32(0.05), by_seq, True, f32(scale))
        most = np.abs(want["dlogp"]).max()
        assert most < 3.3e38 < most * every, what
        assert np.isfinite(got["dlogp"]).all() and (np.abs(got["dlogp"] - want["dlogp"]) <= TOL * want["size"]).all(), what
        size = max(want["size"].max() / scale * every, 1.0)
        if abs(want["loss"]) < 3e38:
            assert abs(got["loss"][0] - want["loss"]) <= TOL * max(size, abs(want["loss"]))
        if want["kl"] < 3e38:
            assert abs(got["kl"][0] - want["kl"]) <= 101 * TOL * want["kl"]


@pytest.mark.parametrize("seqs", [0, 3, 40, 3000])
@pytest.mark.parametrize("by_seq", [False, True])
def test_a_batch_without_tokens_and_a_kl_term(seqs, by_seq):
    """Empty arrays have no address, the reference's among them."""
    none = np.zeros(0, np.float32)
    got = run_policy(none, none, none, np.ones(seqs, np.float32), None, np.zeros(seqs + 1, np.int64), kl=0.05, by_seq=by_seq)
    assert got["loss"][0] == 0 and got["kl"][0] == 0 and got["clipped"][0] == 0
