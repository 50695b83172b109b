"""Workspaces of exactly the size that is asked for at addresses of any alignment: no call writes beside them, and results
do not depend on where they lie."""
import pytest
import torch

from paper_2510_16415_amd import binding as B
from tests.test_gpu_training_step import Step

pytestmark = pytest.mark.gpu
FLANK = 1 << 16
SHIFTS = [0, 1, 16, 128, 240, 255]
TYPE = {"bf16": (torch.bfloat16, B.BF16), "f32": (torch.float32, B.F32)}


class At:
    """n bytes that begin `shift` bytes behind a 256-byte boundary, between two flanks that must stay as they are."""

    def __init__(self, n, shift):
        self.buf = torch.full((n + 2 * FLANK + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.lo = FLANK + (-self.buf.data_ptr()) % 256 + shift
        self.ws = self.buf[self.lo:self.lo + n]
        self.ws.fill_(0xFF)
        self.hi = self.lo + n

    def check(self, what):
        torch.cuda.synchronize()
        before, behind = self.buf[:self.lo], self.buf[self.hi:]
        assert (before == 0xA5).all() and (behind == 0xA5).all(), what


def shifted(need, call, outputs, what):
    """`call` with a workspace of `need` bytes at every shift: the same bits in `outputs`, and nothing beside the workspace."""
    first = None
    for shift in SHIFTS:
        for t in outputs:
            t.fill_(7.0)
        w = At(need, shift)
        call(w.ws)
        w.check((what, shift))
        got = [t.clone() for t in outputs]
        first = first or got
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, got)), (what, shift)


def tensors(dtype, gen):
    tt = TYPE[dtype][0]
    return (lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=gen) * std).to(tt)), (lambda *s: torch.empty(s, device="cuda"))


def ckpt_of(X, code, rows, cols):
    g = -(-cols // 32)
    k = B.ckpt(torch.zeros(rows, 32 * g, dtype=torch.int8, device="cuda"), torch.zeros(rows, g, dtype=torch.uint8, device="cuda"))
    B.mecefo_checkpoint_pack(code, X, rows, cols, X.stride(0), k)
    return k


# 128 x 64 values are whole multiples of 256 bytes: the workspace has no byte to spare behind what is unpacked
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,d,f,r,saved,gain", [(128, 64, 136, 8, False, True), (128, 64, 136, 0, True, True), (256, 128, 200, 16, True, False),
                                                (77, 72, 104, 0, False, False), (2048, 512, 344, 16, False, True)])
def test_block_backwards(dtype, b, d, f, r, saved, gain):
    tt, code = TYPE[dtype]
    rnd, new = tensors(dtype, torch.Generator(device="cuda").manual_seed(b + d))
    W, dOut, gamma = (rnd(f, d, std=0.05), rnd(f, d, std=0.05), rnd(d, f, std=0.05)), rnd(b, d), rnd(d) if gain else None
    P = [B.proj(rnd(n, r, std=n ** -0.5)) if r else None for n in (d, d, f)]
    kept = {n: (x, ckpt_of(x, code, b, x.shape[1])) for n, x in (("H", rnd(b, d)), ("G", rnd(b, f)), ("Z", rnd(b, f)))}
    desc, mask = B.make_desc(b, d, f, code), 0 if r else 7
    dX = torch.empty(b, d, dtype=tt, device="cuda")
    grads = [new(d) if gain else None, new(f, d), new(f, d), new(d, f)]
    outputs = [dX] + [t for t in grads if t is not None]
    more = {n: kept[n] for n in ("G", "Z")} if saved else {}
    shifted(B.mecefo_block_ckpt_workspace_bytes(desc, r, r, r),
            lambda ws: B.mecefo_block_bwd_skip_ckpt(desc, kept["H"][1], dOut, gamma, *W, *P, B.SIDE_INPUT, dX, *grads, 0, ws,
                                                    exact_wgrad_mask=mask, **{n: k for n, (_, k) in more.items()}), outputs, "ckpt")
    shifted(B.mecefo_workspace_bytes(desc, r, r, r),
            lambda ws: B.mecefo_block_bwd_skip_ex(desc, kept["H"][0], dOut, gamma, *W, *P, B.SIDE_INPUT, dX, *grads, 0, ws,
                                                  exact_wgrad_mask=mask, **{n: x for n, (x, _) in more.items()}), outputs, "ex")


@pytest.mark.parametrize("loss", ["preference", "policy"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_training_step(dtype, loss):
    s = Step(dtype, loss=loss)
    sizes = {k: g.n for k, g in s.ws.items()}
    first = None
    for shift in SHIFTS:
        s.ws = {k: At(n, shift) for k, n in sizes.items()}
        s.run()
        for k, w in s.ws.items():
            w.check((k, shift))
        got = s.copies()
        first = first or got
        assert all(torch.equal(first[k].view(torch.uint8), got[k].view(torch.uint8)) for k in first), shift


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_stack_forward_refresh_and_head(dtype):
    tt, code = TYPE[dtype]
    batch, seq, heads, d, f, r = 2, 64, 2, 128, 200, 8
    b = batch * seq
    rnd, new = tensors(dtype, torch.Generator(device="cuda").manual_seed(5))
    act = lambda: torch.empty(b, d, dtype=tt, device="cuda")      # noqa: E731
    w = dict(g_attn=rnd(d), g_ffn=rnd(d), **{k: rnd(d, d, std=0.08) for k in ("Wq", "Wk", "Wv", "Wo")}, Wg=rnd(f, d, std=0.08),
             Wu=rnd(f, d, std=0.08), Wd=rnd(d, f, std=0.08))
    desc, attn, X0 = B.make_desc(b, d, f, code), B.make_attn_desc(batch, seq, heads, d), rnd(b, d)
    H, X = [act(), act()], act()
    shifted(B.mecefo_stack_workspace_bytes(desc, attn, r, r, r),
            lambda ws: B.mecefo_stack_fwd_neighbor(desc, attn, B.layer_weights([w, w]), X0, H, X, ws), [X, *H], "stack_fwd_neighbor")
    P, V0 = torch.empty(d, r, dtype=tt, device="cuda"), rnd(d, r)
    shifted(B.mecefo_projection_workspace_bytes(code, f, d, r, 0),
            lambda ws: B.mecefo_projection_refresh(code, w["Wg"], f, d, d, 0, V0, r, r, 2, 1, 1, P, r, ws), [P], "projection_refresh")
    head = B.make_head_desc(b, d, 333, code)
    Wh, labels, lse, logp = rnd(333, d, std=0.1), torch.arange(b, device="cuda"), new(b), new(b)
    shifted(B.mecefo_head_workspace_bytes(head, False),
            lambda ws: B.mecefo_head_logprob_fwd(head, X0, w["g_ffn"], Wh, labels, logp, lse, ws), [logp, lse], "head_fwd")
    c, dX, dg, dW = rnd(b).float(), act(), new(d), new(333, d)
    shifted(B.mecefo_head_workspace_bytes(head, True),
            lambda ws: B.mecefo_head_logprob_bwd(head, X0, w["g_ffn"], Wh, labels, lse, c, dX, dg, dW, 0, ws), [dX, dg, dW], "head_bwd")
