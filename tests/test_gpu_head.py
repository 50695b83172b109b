"""LM head log-probabilities and their gradient against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from paper_2510_16415_amd import inputs as I
from tests.gpu_util import dev, poisoned_ws, relerr, up8

pytestmark = pytest.mark.gpu
CODE = {"bf16": B.BF16, "f32": B.F32}
U32 = 2.0 ** -24      # half a step of fp32
# a norm-wise gate for the gradients.  bf16: dz is rounded once and the result once, at most 2^-8 of a value each; fp32: a
# sum of K terms in another order, far below the gate of the fp32 path
GATE = {"bf16": 2 * 2.0 ** -8, "f32": 1e-5}


def case(b, d, v, dtype, seed=0, skip=0.2, std=0.2):
    rng = np.random.default_rng([seed, b, d, v])
    cast = (lambda x: I.round_to_bf16_grid(x)) if dtype == "bf16" else (lambda x: x.astype(np.float32))
    X, W = cast(rng.standard_normal((b, d))), cast(rng.standard_normal((v, d)) * std)
    labels = rng.integers(0, v, b)
    labels[rng.random(b) < skip] = rng.choice([-1, -100, v, 1 << 40])
    return X, W, labels.astype(np.int64), rng.standard_normal(b).astype(np.float32) / b


def logp_bound(X, W, scale, v):
    """Per row: two products of d terms added in fp32, each term's partial sums rounded at most d times; the sum of v
    exponentials, added in chains of at most v / 32 + 200 positive terms; exp2 and log to a few units of fp32."""
    size = abs(scale) * (np.abs(X.astype(np.float64)) @ np.abs(W.astype(np.float64)).T).max(axis=1)
    return 2 * (X.shape[1] + 8) * U32 * size + (v / 32 + 260) * U32 + 8 * U32 * size


def run_fwd(X, W, labels, dtype, scale=1.0, gamma=None, pad=0, lse=True, stream=None):
    b, d, v = len(X), X.shape[1], len(W)
    ld = d + pad
    desc = B.make_head_desc(b, d, v, CODE[dtype], B.F32, ld, ld, scale)
    logp, L = torch.full((b,), 9.0, device="cuda"), torch.full((b,), 9.0, device="cuda")
    B.mecefo_head_logprob_fwd(desc, dev(X, dtype, ld), None if gamma is None else dev(gamma, dtype), dev(W, dtype, ld),
                              torch.from_numpy(labels).cuda(), logp, L if lse else None,
                              poisoned_ws(B.mecefo_head_workspace_bytes(desc, False)), stream)
    return logp, L


def run_bwd(X, W, labels, L, c, dtype, scale=1.0, gamma=None, pad=0, grad="f32", accumulate=0, fill=0.25):
    b, d, v = len(X), X.shape[1], len(W)
    ld = d + pad
    gt, gcode = (torch.float32, B.F32) if grad == "f32" else (torch.bfloat16, B.BF16)
    desc = B.make_head_desc(b, d, v, CODE[dtype], gcode, ld, ld, scale)
    dX = torch.full((b, ld), 5.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    dW = torch.full((v, ld), fill, dtype=gt, device="cuda")
    dg = None if gamma is None else torch.full((d,), fill, dtype=gt, device="cuda")
    B.mecefo_head_logprob_bwd(desc, dev(X, dtype, ld), None if gamma is None else dev(gamma, dtype), dev(W, dtype, ld),
                              torch.from_numpy(labels).cuda(), L, torch.from_numpy(c).cuda(), dX, dg, dW, accumulate,
                              poisoned_ws(B.mecefo_head_workspace_bytes(desc, True)))
    if pad:
        assert (dX[:, d:] == 5.0).all() and (dW[:, d:] == fill).all()
    f = lambda t: t.float().cpu().numpy().astype(np.float64)      # noqa: E731
    return f(dX[:, :d]), f(dW[:, :d]), None if dg is None else f(dg)


SIZES = [(1, 8, 1), (1, 64, 7), (2, 16, 8), (3, 40, 33), (17, 64, 255), (64, 128, 257), (65, 256, 1000), (130, 72, 4099),
         (300, 512, 2000), (1, 1024, 32000), (77, 256, 8191), (513, 64, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,d,v", SIZES + [(257, 4096, 515)])
def test_forward(b, d, v, dtype):
    X, W, labels, _ = case(b, d, v, dtype)
    logp, L = run_fwd(X, W, labels, dtype)
    want, lse = T.head_fwd(X, W, labels)
    tol = logp_bound(X, W, 1.0, v)
    assert (np.abs(logp.cpu().numpy() - want) <= tol).all() and (np.abs(L.cpu().numpy() - lse) <= tol).all()
    skipped = (labels < 0) | (labels >= v)
    assert (logp.cpu().numpy()[skipped] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_of_odd_width(dtype):
    d = 24 if dtype == "bf16" else 13
    X, W, labels, _ = case(9, d, 50, dtype)
    logp, L = run_fwd(X, W, labels, dtype, pad=8 if dtype == "bf16" else 3, lse=False)
    want, _ = T.head_fwd(X, W, labels)
    assert (np.abs(logp.cpu().numpy() - want) <= logp_bound(X, W, 1.0, 50)).all() and (L == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.25, -1.5, 0.0, 40.0])
def test_scale_and_large_logits(dtype, scale):
    X, W, labels, c = case(66, 128, 300, dtype, std=1.0)      # at 40: logits in the hundreds
    logp, L = run_fwd(X, W, labels, dtype, scale)
    want, lse = T.head_fwd(X, W, labels, scale)
    tol = logp_bound(X, W, scale, 300)
    assert (np.abs(logp.cpu().numpy() - want) <= tol).all() and (np.abs(L.cpu().numpy() - lse) <= tol).all()
    dX, dW, _ = run_bwd(X, W, labels, L, c, dtype, scale)
    wX, wW = T.head_bwd(X, W, labels, c, scale)
    assert np.isfinite(dX).all() and np.isfinite(dW).all()
    if scale == 0.0:
        assert not dX.any() and not dW.any()
    elif scale < 10:
        assert relerr(dX, wX) <= GATE[dtype] and relerr(dW, wW) <= GATE[dtype]
    else:      # a logit of size 3000 is known to 2 d U32 of that: exp() turns it into a relative error of the probabilities
        more = 2 * tol.max()
        assert relerr(dX, wX) <= GATE[dtype] + more and relerr(dW, wW) <= GATE[dtype] + more


@pytest.mark.parametrize("dtype,grad", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("b,d,v", SIZES)
def test_backward(b, d, v, dtype, grad):
    X, W, labels, c = case(b, d, v, dtype, seed=1)
    _, L = run_fwd(X, W, labels, dtype, pad=8)
    dX, dW, _ = run_bwd(X, W, labels, L, c, dtype, pad=8, grad=grad)
    wX, wW = T.head_bwd(X, W, labels, c)
    if v == 1:      # one word: nothing to learn; the product and its log-sum-exp differ by a rounding
        assert np.abs(dX).max() <= 1e-5 and np.abs(dW).max() <= 1e-5
        return
    assert relerr(dX, wX) <= GATE[dtype] and relerr(dW, wW) <= GATE[dtype]
    skipped = (labels < 0) | (labels >= v)
    assert not dX[skipped].any()


@pytest.mark.parametrize("dtype,grad", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_backward_adds_to_its_gradients(dtype, grad):
    X, W, labels, c = case(130, 64, 500, dtype, seed=2)
    gamma = np.ones(64, np.float32)
    _, L = run_fwd(X, W, labels, dtype, gamma=gamma)
    over = run_bwd(X, W, labels, L, c, dtype, gamma=gamma, grad=grad, accumulate=0)
    more = run_bwd(X, W, labels, L, c, dtype, gamma=gamma, grad=grad, accumulate=1)
    step = 2.0 ** -8 if grad == "bf16" else U32      # rounded once more
    assert np.array_equal(over[0], more[0])
    for a, m in zip(over[1:], more[1:]):
        assert (np.abs(m - (a + 0.25)) <= step * (np.abs(a) + np.abs(m) + 0.25)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,d,v", [(1, 64, 40), (70, 256, 300), (300, 2048, 257), (2500, 128, 100), (40, 4104, 70)])
def test_with_a_norm(b, d, v, dtype):
    X, W, labels, c = case(b, d, v, dtype, seed=3, std=d ** -0.5)
    rng = np.random.default_rng(4)
    gamma = I.round_to_bf16_grid(1 + 0.2 * rng.standard_normal(d)) if dtype == "bf16" else (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
    logp, L = run_fwd(X, W, labels, dtype, gamma=gamma)
    x = X.astype(np.float64)
    rs = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + float(np.float32(1e-6)))
    N = x * rs
    U = N * gamma
    if dtype == "bf16":
        U = I.round_to_bf16_grid(U).astype(np.float64)
    want, lse = T.head_fwd(U, W, labels)
    # U is rounded by the kernel and by the oracle from values that differ in the last bits of fp32: now and then one of
    # them goes to the next number, half a step of bf16 (fp32: a few units)
    flip = (2.0 ** -8 if dtype == "bf16" else 8 * U32) * (np.abs(U) @ np.abs(W.astype(np.float64)).T).max(axis=1)
    tol = logp_bound(U, W, 1.0, v) + 2 * flip
    assert (np.abs(logp.cpu().numpy() - want) <= tol).all() and (np.abs(L.cpu().numpy() - lse) <= tol).all()
    dX, dW, dg = run_bwd(X, W, labels, L, c, dtype, gamma=gamma)
    dU, wW = T.head_bwd(U, W, labels, c)
    dN = dU * gamma
    wX = rs * (dN - N * (dN * N).mean(axis=1, keepdims=True))
    # dz, dU and dX are rounded to bf16, 2^-8 each, and dz and dW see a U that is off as above
    gate = 4 * 2.0 ** -8 if dtype == "bf16" else 1e-5
    assert relerr(dX, wX) <= gate and relerr(dW, wW) <= gate and relerr(dg, (dU * N).sum(axis=0)) <= gate


def test_tokens_that_are_not_scored_may_carry_anything_in_dlogp():
    X, W, labels, c = case(50, 64, 90, "bf16", seed=5, skip=0.5)
    skipped = (labels < 0) | (labels >= 90)
    assert 0 < skipped.sum() < 50
    _, L = run_fwd(X, W, labels, "bf16")
    clean = run_bwd(X, W, labels, L, np.where(skipped, 0, c).astype(np.float32), "bf16")
    dirty = run_bwd(X, W, labels, L, np.where(skipped, np.nan, c).astype(np.float32), "bf16")
    assert np.array_equal(clean[0], dirty[0]) and np.array_equal(clean[1], dirty[1])
    labels[:] = -1
    none = run_bwd(X, W, labels, L, np.full(50, np.inf, np.float32), "bf16")
    assert not none[0].any() and not none[1].any()


def test_no_tokens_clear_or_keep_the_gradients():
    for accumulate in (0, 1):
        desc = B.make_head_desc(0, 64, 90, B.BF16)
        dW, dg = torch.full((90, 64), 2.0, device="cuda"), torch.full((64,), 2.0, device="cuda")
        W, gamma = torch.zeros(90, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
        B.mecefo_head_logprob_bwd(desc, None, gamma, W, None, None, None, None, dg, dW, accumulate,
                                  poisoned_ws(B.mecefo_head_workspace_bytes(desc, True)))
        assert (dW == 2.0 * accumulate).all() and (dg == 2.0 * accumulate).all()


@pytest.mark.parametrize("tile", ["S", "S4", "T", "T2", "X", "L8", "LT", "K", "L4", "L8R"])
def test_every_tile_gives_the_same_to_a_rounding(tile, mecefo_option):
    X, W, labels, c = case(333, 192, 1111, "bf16", seed=6)
    mecefo_option("tile", tile)
    logp, L = run_fwd(X, W, labels, "bf16")
    want, lse = T.head_fwd(X, W, labels)
    tol = logp_bound(X, W, 1.0, 1111)
    assert (np.abs(logp.cpu().numpy() - want) <= tol).all() and (np.abs(L.cpu().numpy() - lse) <= tol).all()
    dX, dW, _ = run_bwd(X, W, labels, L, c, "bf16")
    wX, wW = T.head_bwd(X, W, labels, c)
    assert relerr(dX, wX) <= GATE["bf16"] and relerr(dW, wW) <= GATE["bf16"]


@pytest.mark.parametrize("tile", ["LT", "auto"])
@pytest.mark.parametrize("b,d,v,scale", [(1100, 136, 16563, 1.0), (1280, 192, 13500, -0.7), (261, 1024, 35000, 1.0)])
def test_a_short_last_round_that_is_cut_up(b, d, v, scale, tile, mecefo_option):
    """More than a round of large tiles, and few in the last one; rows that end in the first half of a tile."""
    X, W, labels, c = case(b, d, v, "bf16", seed=13, std=d ** -0.5)
    mecefo_option("tile", tile)
    mecefo_option("head", "all")
    logp, L = run_fwd(X, W, labels, "bf16", scale)
    want, lse = T.head_fwd(X, W, labels, scale)
    tol = logp_bound(X, W, scale, v)
    assert (np.abs(logp.cpu().numpy() - want) <= tol).all() and (np.abs(L.cpu().numpy() - lse) <= tol).all()
    dX, dW, _ = run_bwd(X, W, labels, L, c, "bf16", scale)
    wX, wW = T.head_bwd(X, W, labels, c, scale)
    assert relerr(dX, wX) <= GATE["bf16"] and relerr(dW, wW) <= GATE["bf16"]


@pytest.mark.parametrize("dtype,grad,gamma", [("bf16", "f32", False), ("bf16", "bf16", True), ("f32", "f32", False), ("f32", "f32", True)])
@pytest.mark.parametrize("b,d,v", [(6000, 64, 40), (5000, 72, 257), (9001, 16, 3)])
def test_many_tokens_and_a_small_vocabulary(b, d, v, dtype, grad, gamma):
    """dW cut along the tokens; strides, and a gradient that is added to."""
    X, W, labels, c = case(b, d, v, dtype, seed=21)
    g = np.ones(d, np.float32) if gamma else None
    x = X.astype(np.float64)
    U = x / np.sqrt((x * x).mean(axis=1, keepdims=True) + float(np.float32(1e-6))) if gamma else x
    if gamma and dtype == "bf16":
        U = I.round_to_bf16_grid(U).astype(np.float64)
    _, L = run_fwd(X, W, labels, dtype, gamma=g, pad=8)
    _, dW, _ = run_bwd(X, W, labels, L, c, dtype, gamma=g, pad=8, grad=grad)
    wW = T.head_bwd(U, W, labels, c)[1]
    gate = 4 * 2.0 ** -8 if gamma and dtype == "bf16" else GATE[dtype]      # as with a norm elsewhere
    assert relerr(dW, wW) <= gate
    more = run_bwd(X, W, labels, L, c, dtype, gamma=g, pad=8, grad=grad, accumulate=1)[1]
    step = 2.0 ** -8 if grad == "bf16" else U32
    assert (np.abs(more - (dW + 0.25)) <= step * (np.abs(dW) + np.abs(more) + 0.25)).all()


def test_repeats_are_bit_equal_and_streams_do_not_mix():
    X, W, labels, c = case(200, 256, 3000, "bf16", seed=7)
    first = run_fwd(X, W, labels, "bf16")
    grads = run_bwd(X, W, labels, first[1], c, "bf16")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(run_fwd(X, W, labels, "bf16", stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, first))
    again = run_bwd(X, W, labels, first[1], c, "bf16")
    assert all(np.array_equal(a, b) for a, b in zip(grads[:2], again[:2]))


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("skip", [0.0, 0.3, 0.9, 1.0])
@pytest.mark.parametrize("b,d,v", [(1, 16, 9), (5, 40, 33), (64, 128, 257), (257, 64, 1000), (700, 256, 515), (8300, 16, 40)])
def test_backward_by_the_list_of_scored_rows(b, d, v, skip, grad, mecefo_option):
    X, W, labels, c = case(b, d, v, "bf16", seed=8, skip=skip)
    c[::7] = 0.0      # a label, and no gradient
    mecefo_option("head", "scored")
    _, L = run_fwd(X, W, labels, "bf16", pad=8)
    out = ((labels < 0) | (labels >= v)) | (c == 0)
    dX, dW, _ = run_bwd(X, W, labels, L, c, "bf16", pad=8, grad=grad)
    wX, wW = T.head_bwd(X, W, labels, c)
    assert not dX[out].any()
    assert relerr(dX, wX) <= GATE["bf16"] and relerr(dW, wW) <= GATE["bf16"]
    over, more = dW, run_bwd(X, W, labels, L, c, "bf16", pad=8, grad=grad, accumulate=1)[1]
    step = 2.0 ** -8 if grad == "bf16" else U32
    assert (np.abs(more - (over + 0.25)) <= step * (np.abs(over) + np.abs(more) + 0.25)).all()


@pytest.mark.parametrize("tile", ["S", "S4", "T", "T2", "X", "L8", "LT", "K"])
@pytest.mark.parametrize("b,d,v", [(333, 192, 1111), (600, 512, 700)])
def test_the_list_on_every_tile(tile, b, d, v, mecefo_option):
    X, W, labels, c = case(b, d, v, "bf16", seed=9, skip=0.4)
    mecefo_option("head", "scored")
    mecefo_option("tile", tile)
    _, L = run_fwd(X, W, labels, "bf16")
    dX, dW, _ = run_bwd(X, W, labels, L, c, "bf16")
    wX, wW = T.head_bwd(X, W, labels, c)
    assert relerr(dX, wX) <= GATE["bf16"] and relerr(dW, wW) <= GATE["bf16"]


@pytest.mark.parametrize("tile", ["auto", "LT"])
@pytest.mark.parametrize("scored,v", [(1100, 16563), (1024, 16563), (513, 24000), (1100, 13500), (1281, 13570), (20, 16563), (0, 16563), (900, 16384)])
def test_the_last_round_of_as_many_rows_as_are_listed(scored, v, tile, mecefo_option):
    """Large tiles of the listed rows: rounds with nothing behind them, with a few tiles, with more than half a round, or not a whole one."""
    b, d = max(1100, scored), 72
    X, W, labels, c = case(b, d, v, "bf16", seed=15, skip=0.0, std=d ** -0.5)
    labels[np.random.default_rng(scored).permutation(b)[scored:]] = -1
    mecefo_option("head", "scored")
    mecefo_option("tile", tile)
    _, L = run_fwd(X, W, labels, "bf16")
    dX, dW, _ = run_bwd(X, W, labels, L, c, "bf16")
    wX, wW = T.head_bwd(X, W, labels, c)
    assert not dX[labels < 0].any()
    if scored == 0:
        assert not dW.any()
    else:
        assert relerr(dX, wX) <= GATE["bf16"] and relerr(dW, wW) <= GATE["bf16"]


def test_the_list_with_a_norm_and_with_few_long_products(mecefo_option):
    mecefo_option("head", "scored")
    for b, d, v in ((300, 64, 20000), (40, 2048, 4000)):      # dU cut along the vocabulary
        X, W, labels, c = case(b, d, v, "bf16", seed=10, skip=0.5, std=d ** -0.5)
        gamma = I.round_to_bf16_grid(1 + 0.2 * np.random.default_rng(4).standard_normal(d))
        x = X.astype(np.float64)
        rs = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + float(np.float32(1e-6)))
        N = x * rs
        U = I.round_to_bf16_grid(N * gamma).astype(np.float64)
        _, L = run_fwd(X, W, labels, "bf16", gamma=gamma)
        dX, dW, dg = run_bwd(X, W, labels, L, c, "bf16", gamma=gamma)
        dU, wW = T.head_bwd(U, W, labels, c)
        dN = dU * gamma
        gate = 4 * 2.0 ** -8      # as with a norm above
        assert relerr(dX, rs * (dN - N * (dN * N).mean(axis=1, keepdims=True))) <= gate
        assert relerr(dW, wW) <= gate and relerr(dg, (dU * N).sum(axis=0)) <= gate


def test_large_backwards_go_by_the_list_on_their_own(mecefo_option):
    """The rule's two sides on one size: the same gradients, and the workspace of the side that is taken."""
    b, d, v = 1024, 1024, 65600      # 4e11 operations, the line is at 2e11
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, W = ((torch.randn(s, device="cuda", generator=gen) * k).bfloat16() for s, k in (((b, d), 1.0), ((v, d), 0.02)))
    labels = torch.randint(-v // 4, v, (b,), device="cuda", generator=gen)
    c = torch.randn(b, device="cuda", generator=gen)
    desc = B.make_head_desc(b, d, v, B.BF16, B.BF16)
    logp, L = torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    B.mecefo_head_logprob_fwd(desc, X, None, W, labels, logp, L, poisoned_ws(B.mecefo_head_workspace_bytes(desc, False)))
    got, need = {}, {}
    for rows in ("all", "scored", "auto"):
        mecefo_option("head", rows)
        need[rows] = B.mecefo_head_workspace_bytes(desc, True)
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        B.mecefo_head_logprob_bwd(desc, X, None, W, labels, L, c, dX, None, dW, 0, poisoned_ws(need[rows]))
        got[rows] = (dX.float(), dW.float())
    assert need["auto"] == need["scored"] > need["all"]
    z = X.double() @ W.double().t()
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)).neg_()
    on = labels >= 0
    p[torch.arange(b, device="cuda"), labels.clamp(min=0)] += on.double()
    p *= (c.double() * on)[:, None]
    for dX, dW in got.values():
        for x, y in ((dX, p @ W.double()), (dW, p.t() @ X.double())):
            assert float((x.double() - y).norm() / y.norm()) <= GATE["bf16"]
    assert all(torch.equal(a, s) for a, s in zip(got["auto"], got["scored"]))


def test_a_graph_follows_the_labels_of_its_replays(mecefo_option):
    B.mecefo_init()
    mecefo_option("head", "scored")
    b, d, v = 300, 128, 700
    X, W, labels, c = case(b, d, v, "bf16", seed=11, skip=0.0)
    desc = B.make_head_desc(b, d, v, B.BF16)
    t = dict(X=dev(X, "bf16"), W=dev(W, "bf16"), labels=torch.from_numpy(labels).cuda(), c=torch.from_numpy(c).cuda(),
             logp=torch.empty(b, device="cuda"), L=torch.empty(b, device="cuda"), dX=torch.empty(b, d, dtype=torch.bfloat16, device="cuda"),
             dW=torch.empty(v, d, device="cuda"))
    ws = [poisoned_ws(B.mecefo_head_workspace_bytes(desc, k)) for k in (False, True)]

    def run():
        s = torch.cuda.current_stream()
        B.mecefo_head_logprob_fwd(desc, t["X"], None, t["W"], t["labels"], t["logp"], t["L"], ws[0], s)
        B.mecefo_head_logprob_bwd(desc, t["X"], None, t["W"], t["labels"], t["L"], t["c"], t["dX"], None, t["dW"], 0, ws[1], s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    rng = np.random.default_rng(12)
    for share in (0.0, 0.5, 1.0, 0.97, 0.1):
        now = np.where(rng.random(b) < share, -1, labels)
        t["labels"].copy_(torch.from_numpy(now))
        graph.replay()
        torch.cuda.synchronize()
        wX, wW = T.head_bwd(X, W, now, c)
        assert relerr(t["dX"].float().cpu().numpy(), wX) <= GATE["bf16"] and relerr(t["dW"].cpu().numpy(), wW) <= GATE["bf16"]
        got = [x.clone() for x in (t["dX"], t["dW"])]
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, x) for a, x in zip(got, (t["dX"], t["dW"])))


def test_forward_of_more_logits_than_2_gib():
    """b V logits of 2.3 GB that are not stored; a sample of the rows, the last ones among them."""
    b, d, v = 16411, 64, 70003
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(b, d, device="cuda", generator=gen).bfloat16()
    W = (torch.randn(v, d, device="cuda", generator=gen) * 0.2).bfloat16()
    labels = torch.randint(0, v, (b,), device="cuda", generator=gen)
    labels[-1] = v - 1
    desc = B.make_head_desc(b, d, v, B.BF16, B.F32)
    logp, L = torch.full((b,), 9.0, device="cuda"), torch.full((b,), 9.0, device="cuda")
    B.mecefo_head_logprob_fwd(desc, X, None, W, labels, logp, L, poisoned_ws(B.mecefo_head_workspace_bytes(desc, False)))
    rows = torch.cat([torch.arange(0, b, 797), torch.arange(b - 20, b)])
    x, w = (t.float().cpu().numpy() for t in (X[rows.cuda()], W))
    want, lse = T.head_fwd(x, w, labels.cpu()[rows].numpy())
    tol = logp_bound(x, w, 1.0, v)
    assert (np.abs(logp.cpu()[rows].numpy() - want) <= tol).all() and (np.abs(L.cpu()[rows].numpy() - lse) <= tol).all()


@pytest.mark.parametrize("accumulate", [0, 1])
def test_weight_gradient_beyond_2_gib(accumulate):
    """An fp32 dW of 2.2 GB: rows at both ends, and around 2 GiB."""
    b, d, v = 96, 512, 1060003
    gen = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn(b, d, device="cuda", generator=gen).bfloat16()
    W = (torch.randn(v, d, device="cuda", generator=gen) * 0.1).bfloat16()
    at = (1 << 31) // (4 * d)
    rows = torch.cat([torch.arange(0, 40), torch.arange(at - 40, at + 40), torch.arange(v - 40, v)]).cuda()
    labels = rows[torch.randint(0, len(rows), (b,), device="cuda", generator=gen)]
    labels[-1] = v - 1
    c = torch.randn(b, device="cuda", generator=gen)
    desc = B.make_head_desc(b, d, v, B.BF16, B.F32)
    z = torch.cat([X.double() @ W[i:i + 65536].double().T for i in range(0, v, 65536)], 1)
    lse = torch.logsumexp(z, 1)
    dz = -torch.exp(z - lse[:, None])
    dz[torch.arange(b), labels] += 1.0
    dz *= c.double()[:, None]
    dX, dW = torch.full((b, d), 5.0, device="cuda").bfloat16(), torch.full((v, d), 0.25, device="cuda")
    B.mecefo_head_logprob_bwd(desc, X, None, W, labels, lse.float(), c, dX, None, dW, accumulate,
                              poisoned_ws(B.mecefo_head_workspace_bytes(desc, True)))
    want = dz[:, rows].T @ X.double()
    got = dW[rows].double() - (0.25 if accumulate else 0.0)
    # 0.25 + the gradient is rounded to fp32 where it is added to
    assert (got - want).norm() <= GATE["bf16"] * want.norm() + accumulate * U32 * (0.25 + want.abs().max()) * want.numel() ** 0.5
    wx = torch.zeros(b, d, dtype=torch.float64, device="cuda")
    for i in range(0, v, 65536):
        wx += dz[:, i:i + 65536] @ W[i:i + 65536].double()
    assert (dX.double() - wx).norm() <= GATE["bf16"] * wx.norm()
