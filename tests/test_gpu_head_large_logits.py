"""Logits as large as fp32 holds: a small temperature, or large weights."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from tests.test_gpu_head import U32, case, logp_bound, run_bwd, run_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e5, 1e7, -1e8, 1e9, 3e10, -1e12, 1e20, 1e30, -1e34])
@pytest.mark.parametrize("b,d,v", [(5, 40, 33), (130, 64, 1000), (300, 512, 2000)])
def test_large_logits(b, d, v, scale, dtype):
    X, W, labels, c = case(b, d, v, dtype, seed=31)
    scale = float(np.float32(scale))
    logp, L = (t.cpu().numpy().astype(np.float64) for t in run_fwd(X, W, labels, dtype, scale))
    want, lse = T.head_fwd(X, W, labels, scale)
    tol = logp_bound(X, W, scale, v)
    assert (np.abs(L - lse) <= tol).all() and (np.abs(logp - want) <= tol).all()
    dX, dW, _ = run_bwd(X, W, labels, torch.from_numpy(L.astype(np.float32)).cuda(), c, dtype, scale)
    # which of exp(z - lse) of the largest logits is 1 is beyond what fp32 holds of either; each is at most 1
    on = (labels >= 0) & (labels < v)
    most = abs(scale) * np.abs(c) * on
    reach = 1.01 * most[:, None] * (np.abs(W).max(axis=0) * v)[None, :]
    assert (np.abs(dX) <= reach).all() and (np.abs(dW) <= 1.01 * (most[:, None] * np.abs(X)).sum(axis=0)[None, :]).all()
    assert not dX[~on].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sure_word_has_no_gradient(dtype):
    """One logit far above the others, of a size that fp32 holds exactly: its probability is 1."""
    b, d, v = 70, 64, 300
    X, W = np.zeros((b, d), np.float32), np.zeros((v, d), np.float32)
    X[:, 0] = 1.0
    W[7, 0] = 1.0
    for scale in (2.0 ** 20, 2.0 ** 33, 2.0 ** 100, 2.0 ** 127):
        labels = np.full(b, 7, np.int64)
        labels[::2] = 9
        logp, L = run_fwd(X, W, labels, dtype, scale)
        off = abs(scale) * 4 * U32      # lse through its base-2 logarithm: two roundings each way
        assert (np.abs(L.cpu().numpy().astype(np.float64) - scale) <= off).all()
        assert (np.abs(logp.cpu().numpy()[1::2]) <= off).all() and (np.abs(logp.cpu().numpy()[::2].astype(np.float64) + scale) <= off).all()
        dX, dW, _ = run_bwd(X, W, labels, torch.full((b,), scale, dtype=torch.float32, device="cuda"), np.full(b, 1e-3, np.float32), dtype, scale)
        assert np.isfinite(dX).all() and np.isfinite(dW).all() and np.abs(dX).max() <= 1.01e-3 * scale


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_a_number_stays_in_its_row(dtype):
    X, W, labels, _ = case(70, 64, 300, dtype, seed=32, skip=0.0)
    X[5, 3] = np.nan
    logp, L = (t.cpu().numpy() for t in run_fwd(X, W, labels, dtype))
    assert np.isnan(logp[5]) and np.isnan(L[5]) and np.isfinite(np.delete(logp, 5)).all() and np.isfinite(np.delete(L, 5)).all()
