"""8-bit checkpoints on the GPU: the bytes are the oracle's, the values exact, and the backward from them is the backward on
the unpacked tensors bit for bit."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from tests.gpu_util import dev, poisoned_ws, up8

pytestmark = pytest.mark.gpu
CODE = {"bf16": B.BF16, "f32": B.F32}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def new_ckpt(rows, cols, ld_q=None, ld_e=None):
    g = -(-cols // 32)
    q = torch.full((rows, ld_q or 32 * g), 0x55, dtype=torch.int8, device="cuda")
    e = torch.full((rows, ld_e or g), 0x55, dtype=torch.uint8, device="cuda")
    return B.ckpt(q, e), q, e


def tensor(x, dtype, ld):
    t = torch.full((x.shape[0], ld), float("nan"), dtype=TYPE[dtype], device="cuda")
    t[:, :x.shape[1]] = torch.from_numpy(x).cuda()
    return t


def values(rng, rows, cols, dtype):
    x = rng.standard_normal((rows, cols)) * 10.0 ** rng.uniform(-8, 8, (rows, 1))
    x[:, rng.random(cols) < 0.05] *= 30
    x = x.astype(np.float32)
    return (x.view(np.uint32) & 0xFFFF0000).view(np.float32) if dtype == "bf16" else x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 15), (2, 16), (5, 17), (7, 31), (4, 32), (3, 33), (17, 129), (300, 700), (2, 5461)])
def test_bytes_and_values_are_the_oracles(dtype, rows, cols):
    rng = np.random.default_rng(rows * 10000 + cols)
    x = values(rng, rows, cols, dtype)
    ld = up8(cols) + 8
    g = -(-cols // 32)
    k, q, e = new_ckpt(rows, cols, 32 * g + 16, g + 3)
    X = tensor(x, dtype, ld)
    B.mecefo_checkpoint_pack(CODE[dtype], X, rows, cols, ld, k)
    want_q, want_e = T.ckpt_pack(x)
    assert np.array_equal(q[:, :32 * g].cpu().numpy(), want_q) and np.array_equal(e[:, :g].cpu().numpy(), want_e)
    assert (q[:, 32 * g:] == 0x55).all() and (e[:, g:] == 0x55).all()
    for out in ("bf16", "f32"):
        Y = torch.full((rows, ld), 7.0, dtype=TYPE[out], device="cuda")
        B.mecefo_checkpoint_unpack(CODE[out], k, rows, cols, Y, ld)
        assert np.array_equal(Y[:, :cols].float().cpu().numpy(), T.ckpt_unpack(want_q, want_e, cols))
        assert (Y[:, cols:] == 7.0).all()


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_fp32_rows_of_any_alignment(shift):
    rng = np.random.default_rng(shift)
    x = values(rng, 6, 75, "f32")
    store = torch.zeros(6 * 77 + 8, dtype=torch.float32, device="cuda")
    X = store[shift:shift + 6 * 77].view(6, 77)
    X[:, :75] = torch.from_numpy(x).cuda()
    k, q, e = new_ckpt(6, 75)
    B.mecefo_checkpoint_pack(B.F32, X, 6, 75, 77, k)
    want_q, want_e = T.ckpt_pack(x)
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(e.cpu().numpy(), want_e)
    X.fill_(3.0)
    B.mecefo_checkpoint_unpack(B.F32, k, 6, 75, X, 77)
    assert np.array_equal(X[:, :75].cpu().numpy(), T.ckpt_unpack(want_q, want_e, 75)) and (X[:, 75:] == 3.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_tiny_huge_infinite_and_nan_groups(dtype):
    big, tiny = float(torch.finfo(TYPE[dtype]).max), float(torch.finfo(TYPE[dtype]).smallest_normal)
    x = np.zeros((8, 64), np.float32)
    x[1, 5], x[1, 40] = big, -big
    x[2, 0], x[2, 1], x[2, 33] = tiny, -tiny * 0.25, tiny * 100
    x[3, 3], x[3, 50] = np.inf, 1.0
    x[4, 9], x[4, 45] = np.nan, -2.0
    x[5, 31], x[5, 32] = -np.inf, 1e-3
    x[6] = np.linspace(-127.5, 127.5, 64)      # halves of a step, and the clamp
    x[7, :32] = -128.0
    if dtype == "bf16":
        x = (x.view(np.uint32) & 0xFFFF0000).view(np.float32)
        x[4, 9] = np.nan
    k, q, e = new_ckpt(8, 64)
    B.mecefo_checkpoint_pack(CODE[dtype], tensor(x, dtype, 64), 8, 64, 64, k)
    want_q, want_e = T.ckpt_pack(x)
    assert np.array_equal(e.cpu().numpy(), want_e) and np.array_equal(q.cpu().numpy(), want_q)
    assert want_e[3].tolist()[0] == 255 and want_e[4].tolist()[0] == 255 and want_e[5].tolist()[0] == 255 and want_e[3, 1] != 255
    Y = torch.zeros(8, 64, dtype=TYPE[dtype], device="cuda")
    B.mecefo_checkpoint_unpack(CODE[dtype], k, 8, 64, Y, 64)
    assert np.array_equal(Y.float().cpu().numpy(), T.ckpt_unpack(want_q, want_e, 64), equal_nan=True)


def rnd(rows, cols, std, dtype, ld=None, gen=None):
    t = torch.full((rows, ld or cols), float("nan"), dtype=TYPE[dtype], device="cuda")
    t[:, :cols] = torch.randn(rows, cols, device="cuda", generator=gen) * std
    return t


@pytest.mark.parametrize("dtype,grad", [("bf16", B.F32), ("bf16", B.BF16), ("f32", B.F32)])
@pytest.mark.parametrize("b,d,f,r,mask,saved,gain", [
    (1, 64, 136, 8, 0, False, True), (33, 64, 200, 16, 0, False, True), (300, 256, 700, 32, 2, True, True),
    (129, 128, 341, 0, 7, True, True), (64, 72, 100, 8, 0, True, False), (2500, 512, 344, 16, 0, False, True),
    (520, 2064, 160, 8, 1, True, True), (5, 8, 9, 1, 0, True, True)])
def test_backward_is_that_on_the_unpacked_tensors(dtype, grad, b, d, f, r, mask, saved, gain):
    gen = torch.Generator(device="cuda").manual_seed(b * 7 + d)
    code, ldf, ldd = CODE[dtype], up8(f) + 8, d + 8
    t = lambda rows, cols, std, ld=None: rnd(rows, cols, std, dtype, ld, gen)      # noqa: E731
    dOut, Wg, Wu, Wd = t(b, d, 1.0, ldd), t(f, d, 0.05, ldd), t(f, d, 0.05, ldd), t(d, f, 0.05, ldf)
    gamma = (1 + 0.1 * torch.randn(d, device="cuda", generator=gen)).to(TYPE[dtype]) if gain else None
    P = [B.proj(t(n, r, n ** -0.5, up8(r)), r) if r and not mask >> i & 1 else None for i, n in enumerate((d, d, f))]
    kept, plain = {}, {}
    for name, cols, ld in (("H", d, ldd), ("G", f, ldf), ("Z", f, ldf)):
        if name != "H" and not saved:
            continue
        k, _, _ = new_ckpt(b, cols)
        B.mecefo_checkpoint_pack(code, t(b, cols, 2.0, ld), b, cols, ld, k)
        X = torch.full((b, ld), float("nan"), dtype=TYPE[dtype], device="cuda")
        B.mecefo_checkpoint_unpack(code, k, b, cols, X, ld)
        kept[name], plain[name] = k, X
    desc = B.make_desc(b, d, f, code, grad, ldd, ldf, ldd, ldf)
    gt = torch.float32 if grad == B.F32 else TYPE[dtype]

    def outputs():
        z = lambda *s, t=gt: torch.full(s, 0.5, dtype=t, device="cuda")      # noqa: E731
        return dict(dX=z(b, ldd, t=TYPE[dtype]), dgamma=z(d) if gain else None, dWg=z(f, ldd), dWu=z(f, ldd), dWd=z(d, ldf))
    for accumulate in (0, 1):
        want, got = outputs(), outputs()
        B.mecefo_block_bwd_skip_ex(desc, plain["H"], dOut, gamma, Wg, Wu, Wd, *P, B.SIDE_INPUT, *want.values(), accumulate,
                                   poisoned_ws(B.mecefo_workspace_bytes(desc, r, r, r)), G=plain.get("G"), Z=plain.get("Z"),
                                   exact_wgrad_mask=mask)
        B.mecefo_block_bwd_skip_ckpt(desc, kept["H"], dOut, gamma, Wg, Wu, Wd, *P, B.SIDE_INPUT, *got.values(), accumulate,
                                     poisoned_ws(B.mecefo_block_ckpt_workspace_bytes(desc, r, r, r)), G=kept.get("G"),
                                     Z=kept.get("Z"), exact_wgrad_mask=mask)
        for n in want:
            if want[n] is not None:
                assert torch.equal(want[n].view(torch.uint8), got[n].view(torch.uint8)), (n, accumulate)
                assert torch.isfinite(got[n].float()).all(), n


def test_backward_in_place_and_of_no_tokens():
    b, d, f = 70, 64, 136
    gen = torch.Generator(device="cuda").manual_seed(5)
    t = lambda rows, cols, std: rnd(rows, cols, std, "bf16", None, gen)      # noqa: E731
    dOut, W = t(b, d, 1.0), (t(f, d, 0.05), t(f, d, 0.05), t(d, f, 0.05))
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    k, _, _ = new_ckpt(b, d)
    B.mecefo_checkpoint_pack(B.BF16, t(b, d, 1.0), b, d, d, k)
    res = []
    for in_place in (False, True):
        g = dOut.clone()
        dX = g if in_place else torch.empty_like(g)
        out = [torch.empty(s, device="cuda") for s in ((d,), (f, d), (f, d), (d, f))]
        desc = B.make_desc(b, d, f, B.BF16)
        B.mecefo_block_bwd_skip_ckpt(desc, k, g, gamma, *W, None, None, None, B.SIDE_INPUT, dX, *out, 0,
                                     poisoned_ws(B.mecefo_block_ckpt_workspace_bytes(desc)), exact_wgrad_mask=7)
        res.append([dX, *out])
    assert all(torch.equal(x, y) for x, y in zip(*res))
    out = [torch.full(s, 3.0, device="cuda") for s in ((d,), (f, d), (f, d), (d, f))]
    desc = B.make_desc(0, d, f, B.BF16)
    none = B.Ckpt(None, None, 64, 2)
    B.mecefo_block_bwd_skip_ckpt(desc, none, None, gamma, *W, None, None, None, B.SIDE_INPUT, None, *out, 0,
                                 poisoned_ws(B.mecefo_block_ckpt_workspace_bytes(desc)), exact_wgrad_mask=7)
    assert all(not t.any() for t in out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,seq,heads,dh,layers", [(2, 40, 2, 64, 3), (1, 1, 1, 16, 1)])
def test_stack_keeps_and_reads_checkpoints(dtype, batch, seq, heads, dh, layers):
    b, d, f, r = batch * seq, heads * dh, 136, 8
    gen = torch.Generator(device="cuda").manual_seed(11)
    code = CODE[dtype]
    t = lambda rows, cols, std: rnd(rows, cols, std, dtype, None, gen)      # noqa: E731
    one = torch.ones(d, dtype=TYPE[dtype], device="cuda")
    W = [dict(g_attn=one, g_ffn=one, **{k: t(d, d, 0.1) for k in ("Wq", "Wk", "Wv", "Wo")}, Wg=t(f, d, 0.1), Wu=t(f, d, 0.1),
              Wd=t(d, f, 0.1)) for _ in range(layers)]
    lw = B.layer_weights(W)
    desc, attn = B.make_desc(b, d, f, code), B.make_attn_desc(batch, seq, heads, d)
    X0, top = t(b, d, 1.0), t(b, d, 1.0)
    act = lambda: torch.empty(b, d, dtype=TYPE[dtype], device="cuda")      # noqa: E731
    H, X1, X2 = [act() for _ in W], act(), act()
    B.mecefo_stack_fwd_neighbor(desc, attn, lw, X0, H, X1, poisoned_ws(B.mecefo_stack_workspace_bytes(desc, attn, r, r, r)))
    ks = [new_ckpt(b, d) for _ in W]
    kept = B.ckpt_array([k for k, _, _ in ks])
    ws = poisoned_ws(B.mecefo_stack_ckpt_workspace_bytes(desc, attn, r, r, r))
    B.mecefo_stack_fwd_neighbor_ckpt(desc, attn, lw, X0, kept, X2, ws)
    assert torch.equal(X1, X2)
    back = []
    for h, (_, q, e) in zip(H, ks):
        want_q, want_e = T.ckpt_pack(h.float().cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(e.cpu().numpy(), want_e)
        back.append(torch.from_numpy(T.ckpt_unpack(want_q, want_e, d)).cuda().to(TYPE[dtype]))
    proj = [[t(n, r, n ** -0.5) for n in (d, d, f)] for _ in W]
    res = []
    for which in (0, 1):
        low = [dict(Pg=B.proj(p[0]), Pu=B.proj(p[1]), Pd=B.proj(p[2]),
                    **{k: torch.zeros(s, device="cuda") for k, s in (("dg_ffn", (d,)), ("dWg", (f, d)), ("dWu", (f, d)), ("dWd", (d, f)))})
               for p in proj]
        dX = act()
        if which == 0:
            B.mecefo_stack_bwd_skip(desc, lw, back, B.layer_lowrank(low), B.SIDE_INPUT, top, dX, 0,
                                    poisoned_ws(B.mecefo_stack_workspace_bytes(desc, attn, r, r, r)))
        else:
            B.mecefo_stack_bwd_skip_ckpt(desc, lw, kept, B.layer_lowrank(low), B.SIDE_INPUT, top, dX, 0, ws)
        res.append([dX] + [q[k] for q in low for k in ("dg_ffn", "dWg", "dWu", "dWd")])
    assert all(torch.equal(x, y) for x, y in zip(*res))
