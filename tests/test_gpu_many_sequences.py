"""Losses over batches of many short sequences: against the oracle, and in a time that grows with the batch and not with its square."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from tests.test_gpu_loss import ONCE, arrays, check_policy, check_preference, cu, f32, loss_size, offsets, run_policy, run_preference, spoil

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("seqs,mean_len", [(1025, 2), (2048, 3), (2049, 3), (5000, 1), (70000, 1)])
def test_many_sequences(seqs, mean_len, masked):
    rng = np.random.default_rng([seqs, mean_len, int(masked * 10)])
    off = offsets(rng, seqs, mean_len, front=int(rng.integers(0, 3)), empty=0.2)
    lp, old, r, mask = arrays(rng, int(off[-1]) + 5, masked)
    for by_seq, per_token in ((False, True), (True, False)):
        adv = rng.standard_normal(len(lp) if per_token else seqs).astype(np.float32)
        got = run_policy(spoil(lp, mask, rng), spoil(old, mask, rng), spoil(r, mask, rng), adv, mask, off, kl=0.05, by_seq=by_seq, per_token=per_token)
        want = T.policy(lp, old, r, adv, mask, off, f32(0.2), f32(0.28), f32(0.05), by_seq, per_token)
        check_policy(got, want, loss_size(lp, old, r, adv, mask, off, 0.05, by_seq, per_token))
    if seqs % 2 == 0:
        got = run_preference(spoil(lp, mask, rng), spoil(r, mask, rng), mask, off, 0.3)
        check_preference(got, T.preference(lp, r, mask, off, f32(0.3), 0.0, 0.0, False))


def test_many_sequences_without_a_counted_token():
    off = np.arange(3001, dtype=np.int64) * 2
    for by_seq in (False, True):
        got = run_policy(np.full(6001, np.nan, np.float32), np.zeros(6001, np.float32), None, np.ones(3000, np.float32),
                         np.zeros(6001, np.uint8), off, by_seq=by_seq)
        assert got["loss"][0] == 0 and got["kl"][0] == 0 and got["clipped"][0] == 0 and not got["dlogp"].any()


@pytest.mark.parametrize("by_seq", [False, True])
def test_as_many_sequences_as_are_taken(by_seq):
    """2^20 sequences of 3 tokens.  The call takes 4 ms; where every workgroup reads the counts of all sequences it is above 300."""
    n, rng = 1 << 20, np.random.default_rng(int(by_seq))
    lp, old, r, _ = arrays(rng, 3 * n, 0.0)
    adv = rng.standard_normal(n).astype(np.float32)
    desc = B.make_policy_desc(3 * n, n, 0.2, 0.28, 0.05, B.MEAN_SEQUENCES if by_seq else B.MEAN_TOKENS)
    t = [cu(x) for x in (lp, old, r, adv)]
    off, loss, dlogp = torch.arange(n + 1, device="cuda") * 3, torch.zeros(1, device="cuda"), torch.zeros(3 * n, device="cuda")
    ws = torch.full((B.mecefo_policy_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    times = []
    for _ in range(3):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        B.mecefo_policy_loss(desc, *t, None, off, loss, None, None, dlogp, ws)
        end.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(end))
    d, A = lp.astype(np.float64) - old, np.repeat(adv.astype(np.float64), 3)
    q = r.astype(np.float64) - lp
    rho = np.exp(d)
    kept = np.clip(rho, 1 - f32(0.2), 1 + f32(0.28))
    over = kept * A < rho * A
    terms = f32(0.05) * (np.expm1(q) - q) - np.minimum(rho * A, kept * A)
    grad = np.where(over, 0.0, -rho * A) - f32(0.05) * np.expm1(q)      # equal lengths: the same weight for all
    tol = 16 * 2.0 ** -24      # as in check_policy
    size = rho * np.abs(A) * (1 + np.abs(d)) + f32(0.05) * np.abs(np.expm1(q))
    assert (np.abs(dlogp.cpu().numpy() * (3.0 * n) - grad) <= tol * size).all()
    assert abs(float(loss) - terms.mean()) <= tol * np.abs(terms).mean() + ONCE * abs(terms.mean())
    assert min(times) < 60, times
