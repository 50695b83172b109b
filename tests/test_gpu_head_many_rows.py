"""The head over as many rows as its operands' sizes allow: more than a launch has workgroups of 1024 threads."""
import pytest
import torch

from paper_2510_16415_amd import binding as B
from tests.gpu_util import poisoned_ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,d,v", [((1 << 22) + 3, 8, 5), (5000001, 16, 40)])
def test_forward_and_backward(b, d, v, dtype):
    tt, code = (torch.float32, B.F32) if dtype == "f32" else (torch.bfloat16, B.BF16)
    gen = torch.Generator(device="cuda").manual_seed(2)
    X, W = torch.randn(b, d, device="cuda", generator=gen).to(tt), (torch.randn(v, d, device="cuda", generator=gen) * 0.3).to(tt)
    labels = torch.randint(-1, v, (b,), device="cuda", generator=gen)
    c = torch.randn(b, device="cuda", generator=gen) / b
    desc = B.make_head_desc(b, d, v, code)
    logp, lse = torch.full((b,), 9.0, device="cuda"), torch.full((b,), 9.0, device="cuda")
    B.mecefo_head_logprob_fwd(desc, X, None, W, labels, logp, lse, poisoned_ws(B.mecefo_head_workspace_bytes(desc, False)))
    dX, dW = torch.full((b, d), 5.0, dtype=tt, device="cuda"), torch.full((v, d), 5.0, device="cuda")
    B.mecefo_head_logprob_bwd(desc, X, None, W, labels, lse, c, dX, None, dW, 0, poisoned_ws(B.mecefo_head_workspace_bytes(desc, True)))
    want = torch.zeros(v, d, dtype=torch.float64, device="cuda")
    gate = 2 * 2.0 ** -8 if dtype == "bf16" else 1e-5      # the head tests' gates
    for i in range(0, b, 1 << 20):
        at = slice(i, min(b, i + (1 << 20)))
        z = X[at].double() @ W.double().t()
        l, on = torch.logsumexp(z, 1), labels[at] >= 0
        own = torch.gather(z, 1, labels[at].clamp(min=0)[:, None])[:, 0]
        # sums of 16 products and 40 exponentials in fp32: below 100 half-steps of the largest logit
        tol = 100 * 2.0 ** -24 * (1 + z.abs().max(1).values)
        assert ((lse[at] - l).abs() <= tol).all() and ((logp[at] - torch.where(on, own - l, 0.0)).abs() <= 2 * tol).all(), i
        dz = -torch.exp(z - l[:, None])
        dz[torch.arange(len(z), device="cuda"), labels[at].clamp(min=0)] += 1.0
        dz *= (c[at].double() * on)[:, None]
        dU = dz @ W.double()
        assert (dX[at].double() - dU).norm() <= gate * dU.norm(), i
        want += dz.t() @ X[at].double()
    assert (dW.double() - want).norm() <= gate * want.norm()


@pytest.mark.parametrize("gain", [False, True])
def test_the_most_rows(gain):
    """2^26 - 64 rows of 16 bytes; a sample of them, both ends among it."""
    b, d, v = (1 << 26) - 64, 8, 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.empty(b, d, dtype=torch.bfloat16, device="cuda")
    for i in range(0, b, 1 << 23):
        X[i:i + (1 << 23)] = torch.randn(min(b - i, 1 << 23), d, device="cuda", generator=gen).bfloat16()
    W = torch.randn(v, d, device="cuda", generator=gen).bfloat16()
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda") if gain else None
    labels = torch.randint(0, v, (b,), device="cuda", generator=gen)
    c = torch.randn(b, device="cuda", generator=gen) / b
    desc = B.make_head_desc(b, d, v, B.BF16)
    logp, lse = torch.full((b,), 9.0, device="cuda"), torch.full((b,), 9.0, device="cuda")
    B.mecefo_head_logprob_fwd(desc, X, gamma, W, labels, logp, lse, poisoned_ws(B.mecefo_head_workspace_bytes(desc, False)))
    dX, dW = torch.full((b, d), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((v, d), 5.0, device="cuda")
    dg = torch.full((d,), 5.0, device="cuda") if gain else None
    B.mecefo_head_logprob_bwd(desc, X, gamma, W, labels, lse, c, dX, dg, dW, 0, poisoned_ws(B.mecefo_head_workspace_bytes(desc, True)))
    at = torch.cat([torch.arange(0, 4096), torch.arange(0, b, 9973), torch.arange(b - 4096, b)]).cuda()
    x = X[at].double()
    rs = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + float(torch.tensor(1e-6, dtype=torch.float32)))
    U = (x * rs).bfloat16().double() if gain else x
    z = U @ W.double().t()
    l = torch.logsumexp(z, 1)
    own = torch.gather(z, 1, labels[at][:, None])[:, 0]
    # with a gain U may be rounded to its neighbour: 2^-8 of a value, each term of eight
    tol = 100 * 2.0 ** -24 * (1 + z.abs().max(1).values) + (2.0 ** -7 * (U.abs() @ W.double().abs().t()).max(1).values if gain else 0.0)
    assert ((lse[at] - l).abs() <= tol).all() and ((logp[at] - (own - l)).abs() <= 2 * tol).all()
    dz = -torch.exp(z - l[:, None])
    dz[torch.arange(len(z), device="cuda"), labels[at]] += 1.0
    dU = (dz * c[at].double()[:, None]) @ W.double()
    N = x * rs
    want = rs * (dU - N * (dU * N).mean(1, keepdim=True)) if gain else dU
    gate = (4 if gain else 2) * 2.0 ** -8
    assert (dX[at].double() - want).norm() <= gate * want.norm() and torch.isfinite(dW).all()
