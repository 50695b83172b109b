"""Preference and policy loss against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from tests.gpu_util import poisoned_ws

pytestmark = pytest.mark.gpu
# results are formed in fp64 from fp32 inputs and rounded once; exp and log1p of either library to a few units of fp64
ONCE = 2.0 ** -23


def offsets(rng, n, mean, front=0, empty=0.1):
    lens = np.where(rng.random(n) < empty, 0, rng.integers(0, 2 * mean + 1, n))
    return (front + np.concatenate([[0], np.cumsum(lens)])).astype(np.int64)


def arrays(rng, tokens, masked):
    lp = (-3 * rng.random(tokens)).astype(np.float32)
    near = lambda s: (lp + s * rng.standard_normal(tokens)).astype(np.float32)      # noqa: E731
    mask = (rng.random(tokens) > masked).astype(np.uint8) * rng.integers(1, 256, tokens).astype(np.uint8) if masked else None
    return lp, near(0.3), near(0.2), mask


def cu(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def out(n):
    return torch.full((max(n, 1),), 9.0, device="cuda")[:n]


def spoil(x, mask, rng):
    """What does not count may hold anything."""
    if mask is None:
        return x
    bad = rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38, np.finfo(np.float32).min], np.float32), len(x))
    return np.where(mask > 0, x, bad).astype(np.float32)


def run_preference(lp, ref, mask, off, beta, smooth=0.0, margin=0.0, mean=False, grad_scale=1.0, extras=True, stream=None):
    n = (len(off) - 1) // 2
    desc = B.make_preference_desc(len(lp), n, beta, smooth, margin, mean, grad_scale)
    o = dict(loss=out(1), margins=out(n), rewards=out(2 * n), dlogp=out(len(lp)))
    B.mecefo_preference_loss(desc, cu(lp), cu(ref), cu(mask), cu(off), o["loss"], o["margins"] if extras else None,
                             o["rewards"] if extras else None, o["dlogp"],
                             poisoned_ws(B.mecefo_preference_workspace_bytes(desc)), stream)
    return {k: v.cpu().numpy().astype(np.float64) for k, v in o.items()}


def f32(x):
    return float(np.float32(x))


def check_preference(got, want):
    # the loss and the slopes see h, itself a difference of sums: its fp64 error is far below ONCE
    assert abs(got["loss"][0] - want["loss"]) <= ONCE * abs(want["loss"])
    for k in ("margins", "rewards", "dlogp"):
        assert (np.abs(got[k] - want[k]) <= ONCE * np.abs(want[k]) + 1e-12).all(), k


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("pairs,mean_len", [(1, 1), (1, 3), (3, 20), (2, 700), (40, 6), (1, 9000), (5, 3001), (300, 2)])
@pytest.mark.parametrize("ref,mean,smooth,margin", [(True, False, 0.0, 0.0), (False, True, 0.1, 0.5)])
def test_preference(pairs, mean_len, ref, mean, smooth, margin, masked):
    rng = np.random.default_rng([pairs, mean_len, int(mean), int(masked * 10)])
    off = offsets(rng, 2 * pairs, mean_len, front=int(rng.integers(0, 3)))
    lp, _, r, mask = arrays(rng, int(off[-1]) + int(rng.integers(0, 4)), masked)
    beta = 2.0 if mean else 0.3 / np.sqrt(mean_len)
    got = run_preference(spoil(lp, mask, rng), spoil(r, mask, rng) if ref else None, mask, off, beta, smooth, margin, mean)
    check_preference(got, T.preference(lp, r if ref else None, mask, off, f32(beta), f32(smooth), f32(margin), mean))


def test_preference_of_sure_pairs_and_scaled_gradients():
    off = np.array([0, 2, 4, 6, 8], np.int64)
    lp = np.array([0, 0, -300, -300, -300, -300, 0, 0], np.float32)      # h = +600 and -600
    got = run_preference(lp, None, None, off, 1.0, grad_scale=-8.0, extras=False)
    want = T.preference(lp, None, None, off, 1.0, grad_scale=-8.0)
    assert got["loss"][0] == 300.0 and np.array_equal(got["dlogp"], want["dlogp"].astype(np.float32).astype(np.float64))
    assert (got["margins"] == 9.0).all() and (got["rewards"] == 9.0).all()


def test_preference_without_pairs_or_tokens():
    got = run_preference(np.ones(5, np.float32), None, None, np.zeros(1, np.int64), 0.1)
    assert got["loss"][0] == 0 and not got["dlogp"].any()
    got = run_preference(np.zeros(0, np.float32), None, None, np.zeros(5, np.int64), 0.1)
    assert got["loss"][0] == pytest.approx(np.log(2), rel=ONCE) and not got["margins"].any()
    got = run_preference(np.full(6, np.nan, np.float32), None, np.zeros(6, np.uint8), np.array([0, 3, 6], np.int64), 0.1, mean=True)
    assert got["loss"][0] == pytest.approx(np.log(2), rel=ONCE) and not got["dlogp"].any()


def run_policy(lp, old, ref, adv, mask, off, low=0.2, high=0.28, kl=0.0, by_seq=False, per_token=False, grad_scale=1.0, extras=True):
    desc = B.make_policy_desc(len(lp), len(off) - 1, low, high, kl, B.MEAN_SEQUENCES if by_seq else B.MEAN_TOKENS, per_token, grad_scale)
    o = dict(loss=out(1), kl=out(1), clipped=out(1), dlogp=out(len(lp)))
    B.mecefo_policy_loss(desc, cu(lp), cu(old), cu(ref), cu(adv), cu(mask), cu(off), o["loss"], o["kl"] if extras else None,
                         o["clipped"] if extras else None, o["dlogp"], poisoned_ws(B.mecefo_policy_workspace_bytes(desc)))
    return {k: v.cpu().numpy().astype(np.float64) for k, v in o.items()}


def check_policy(got, want, loss_size):
    # a token's terms: the difference of two fp32 numbers rounded to fp32 (2^-24 of it, an error of as much in its exp), expf and
    # expm1f to two units, four products: at most 16 half-steps of fp32 of their size; the sums in fp64
    tol = 16 * 2.0 ** -24
    assert (np.abs(got["dlogp"] - want["dlogp"]) <= tol * want["size"]).all()
    assert abs(got["loss"][0] - want["loss"]) <= tol * loss_size
    assert abs(got["kl"][0] - want["kl"]) <= tol * want["kl"]
    assert abs(got["clipped"][0] - want["clipped"]) <= ONCE


def loss_size(lp, old, ref, adv, mask, off, kl, by_seq, per_token):
    """The loss with every term taken by its size, the ratio at its largest."""
    a = np.abs(adv).max() if len(adv) else 0.0
    spread = np.abs(lp.astype(np.float64) - old).max() if len(lp) else 0.0
    return (1 + spread) * np.exp(min(spread, 50)) * a + kl * (np.exp(np.abs(lp.astype(np.float64) - ref).max()) if ref is not None and len(lp) else 0.0)


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("seqs,mean_len", [(1, 1), (3, 2), (7, 30), (2, 5000), (100, 11), (1, 20000), (600, 3)])
@pytest.mark.parametrize("ref,by_seq,per_token", [(True, False, True), (True, True, False), (False, True, True)])
def test_policy(seqs, mean_len, ref, by_seq, per_token, masked):
    rng = np.random.default_rng([seqs, mean_len, int(by_seq), int(masked * 10), int(ref)])
    off = offsets(rng, seqs, mean_len, front=int(rng.integers(0, 3)))
    lp, old, r, mask = arrays(rng, int(off[-1]) + int(rng.integers(0, 4)), masked)
    adv = rng.standard_normal(len(lp) if per_token else seqs).astype(np.float32)
    kl = 0.05 if ref else 0.0
    r = r if ref else None
    got = run_policy(spoil(lp, mask, rng), spoil(old, mask, rng), spoil(r, mask, rng) if ref else None,
                     spoil(adv, mask, rng) if per_token else adv, mask, off, kl=kl, by_seq=by_seq, per_token=per_token)
    want = T.policy(lp, old, r, adv, mask, off, f32(0.2), f32(0.28), f32(kl), by_seq, per_token)
    check_policy(got, want, loss_size(lp, old, r, adv, mask, off, kl, by_seq, per_token))


def test_policy_on_its_bounds():
    # differences next to log(1 + high) and log(1 - low), as fp32 holds them, on either side
    low, high = f32(0.2), f32(0.28)
    up_, down = np.float32(np.log1p(high)), np.float32(np.log1p(-low))
    lp = np.array([up_, np.nextafter(up_, np.float32(1)), np.nextafter(up_, np.float32(0)), down, np.nextafter(down, np.float32(-1)),
                   np.nextafter(down, np.float32(0)), 0, 0], np.float32)
    old = np.zeros(8, np.float32)
    for sign in (1.0, -1.0):
        adv = np.full(8, sign, np.float32)
        got = run_policy(lp, old, None, adv, None, np.array([0, 8], np.int64), low, high, per_token=True)
        diff = lp.astype(np.float64)
        over = diff > np.log1p(high) if sign > 0 else diff < np.log1p(-low)
        assert 0 < over.sum() < 3
        assert np.array_equal(got["dlogp"] == 0, over) and got["clipped"][0] == over.sum() / 8


def test_policy_that_clips_everything_or_nothing():
    rng = np.random.default_rng(8)
    lp, old, ref, _ = arrays(rng, 50, 0.0)
    adv = rng.standard_normal(50).astype(np.float32)
    off = np.array([0, 50], np.int64)
    got = run_policy(lp, old, None, adv, None, off, low=1.0, high=1e30, per_token=True, grad_scale=2.0, extras=False)
    want = T.policy(lp, old, None, adv, None, off, 1.0, float(np.float32(1e30)), 0.0, False, True, 2.0)
    assert (np.abs(got["dlogp"] - want["dlogp"]) <= 16 * 2.0 ** -24 * want["size"]).all() and got["kl"][0] == 9.0 and got["clipped"][0] == 9.0
    got = run_policy(lp, lp - np.float32(1e-3), None, np.ones(1, np.float32), None, off, low=0.0, high=0.0)
    assert not got["dlogp"].any() and got["clipped"][0] == 1 and got["loss"][0] == -1.0


def test_policy_kl_of_small_differences_keeps_its_digits():
    rng = np.random.default_rng(9)
    lp = (-rng.random(2000)).astype(np.float32)
    ref = (lp.astype(np.float64) + 1e-4 * rng.standard_normal(2000)).astype(np.float32)
    off = np.array([0, 2000], np.int64)
    got = run_policy(lp, lp, ref, np.zeros(1, np.float32), None, off, kl=1.0)
    want = T.policy(lp, lp, ref, np.zeros(1, np.float32), None, off, f32(0.2), f32(0.28), 1.0)
    check_policy(got, want, want["kl"])
    assert got["loss"][0] == got["kl"][0]


def test_policy_of_nothing():
    got = run_policy(np.zeros(4, np.float32), np.zeros(4, np.float32), None, np.zeros(0, np.float32), None, np.zeros(1, np.int64))
    assert got["loss"][0] == 0 and got["clipped"][0] == 0 and not got["dlogp"].any()
    for by_seq in (False, True):
        got = run_policy(np.full(4, np.nan, np.float32), np.zeros(4, np.float32), None, np.ones(2, np.float32), np.zeros(4, np.uint8),
                         np.array([0, 4, 4], np.int64), by_seq=by_seq)
        assert got["loss"][0] == 0 and got["kl"][0] == 0 and not got["dlogp"].any()


def test_repeats_are_bit_equal_on_other_streams():
    rng = np.random.default_rng(10)
    off = offsets(rng, 40, 500)
    lp, old, ref, mask = arrays(rng, int(off[-1]), 0.3)
    first = run_preference(lp, ref, mask, off, 0.01)
    for _ in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            again = run_preference(lp, ref, mask, off, 0.01, stream=s)
        assert all(np.array_equal(first[k], again[k]) for k in first)
    adv = rng.standard_normal(40).astype(np.float32)
    a, b = (run_policy(lp, old, ref, adv, mask, off, kl=0.1, by_seq=True) for _ in range(2))
    assert all(np.array_equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("front,used,behind", [(70001, 900, 60002), (0, 3, 200000), (131073, 0, 0)])
def test_tokens_of_no_sequence_get_zeros(front, used, behind):
    """A buffer that is larger than the batch in it: what lies outside holds NaN and is not looked at."""
    rng = np.random.default_rng([front, used])
    n = front + used + behind
    off = front + np.array([0, used // 3, used // 2, used // 2, used], np.int64)
    inside = np.zeros(n, bool)
    inside[front:front + used] = True
    lp, old, r, _ = arrays(rng, n, 0.0)
    adv = rng.standard_normal(n).astype(np.float32)
    bad = [np.where(inside, x, np.float32(np.nan)) for x in (lp, r, old, adv)]
    check_preference(run_preference(bad[0], bad[1], None, off, 0.02), T.preference(lp, r, None, off, f32(0.02), 0.0, 0.0, False))
    got = run_policy(bad[0], bad[2], bad[1], bad[3], None, off, kl=0.1, by_seq=True, per_token=True)
    check_policy(got, T.policy(lp, old, r, adv, None, off, f32(0.2), f32(0.28), f32(0.1), True, True),
                 loss_size(lp, old, r, adv, None, off, 0.1, True, True))


@pytest.mark.parametrize("seqs,mean_len", [(24, 8200), (4, 33000), (34, 9000)])
def test_few_sequences_of_many_slices(seqs, mean_len):
    rng = np.random.default_rng([seqs, mean_len])
    off = offsets(rng, seqs, mean_len, front=1)
    lp, old, r, mask = arrays(rng, int(off[-1]) + 2, 0.3)
    beta = 0.3 / np.sqrt(mean_len)
    got = run_preference(spoil(lp, mask, rng), spoil(r, mask, rng), mask, off, beta)
    check_preference(got, T.preference(lp, r, mask, off, f32(beta), 0.0, 0.0, False))
    adv = rng.standard_normal(seqs).astype(np.float32)
    for by_seq in (False, True):
        got = run_policy(spoil(lp, mask, rng), spoil(old, mask, rng), spoil(r, mask, rng), adv, mask, off, kl=0.05, by_seq=by_seq)
        check_policy(got, T.policy(lp, old, r, adv, mask, off, f32(0.2), f32(0.28), f32(0.05), by_seq),
                     loss_size(lp, old, r, adv, mask, off, 0.05, by_seq, False))
