"""The new calls as a training step makes them: a neighbor-mode stack that keeps 8-bit checkpoints, the head, a loss, the head's
gradient and the stack's backward from the checkpoints; workspaces of exactly the size that is asked for; captured graphs."""
import numpy as np
import pytest
import torch

from oracle import mecefo_oracle as O
from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from tests.gpu_util import poisoned_ws, relerr

pytestmark = pytest.mark.gpu
FLANK = 1 << 16


class Guarded:
    """A workspace of exactly the size asked for, between two flanks that must stay as they are."""

    def __init__(self, n):
        self.n = n
        self.buf = torch.full((n + 2 * FLANK,), 0xA5, dtype=torch.uint8, device="cuda")
        self.ws = self.buf[FLANK:FLANK + n]

    def check(self, what):
        torch.cuda.synchronize()
        assert (self.buf[:FLANK] == 0xA5).all() and (self.buf[FLANK + self.n:] == 0xA5).all(), what


class Step:
    """One step on `pairs` pairs of answers: buffers, and the calls in order."""

    def __init__(self, dtype="bf16", batch=4, seq=24, heads=2, dh=64, f=136, r=8, layers=2, vocab=301, loss="preference"):
        self.tt = torch.bfloat16 if dtype == "bf16" else torch.float32
        code = B.BF16 if dtype == "bf16" else B.F32
        b, d = batch * seq, heads * dh
        self.b, self.d, self.f, self.layers, self.loss_kind, self.batch = b, d, f, layers, loss, batch
        gen = torch.Generator(device="cuda").manual_seed(3)
        rnd = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=gen) * std).to(self.tt)      # noqa: E731
        new = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device="cuda")      # noqa: E731
        gain = lambda: (1 + 0.1 * torch.randn(d, device="cuda", generator=gen)).to(self.tt)      # noqa: E731
        self.W = [dict(g_attn=gain(), g_ffn=gain(), **{k: rnd(d, d, std=0.08) for k in ("Wq", "Wk", "Wv", "Wo")},
                       Wg=rnd(f, d, std=0.08), Wu=rnd(f, d, std=0.08), Wd=rnd(d, f, std=0.08)) for _ in range(layers)]
        self.P = [[rnd(n, r, std=n ** -0.5) for n in (d, d, f)] for _ in range(layers)]
        self.low = [dict(Pg=B.proj(p[0]), Pu=B.proj(p[1]), Pd=B.proj(p[2]), dg_ffn=new(d), dWg=new(f, d), dWu=new(f, d),
                         dWd=new(d, f)) for p in self.P]
        self.lw, self.lr = B.layer_weights(self.W), B.layer_lowrank(self.low)
        self.desc, self.attn = B.make_desc(b, d, f, code), B.make_attn_desc(batch, seq, heads, d)
        g = d // 32
        self.q = [(torch.zeros(b, 32 * g, dtype=torch.int8, device="cuda"), torch.zeros(b, g, dtype=torch.uint8, device="cuda"))
                  for _ in range(layers)]
        self.H = B.ckpt_array([B.ckpt(*x) for x in self.q])
        self.X0, self.X, self.dX = rnd(b, d), new(b, d, t=self.tt), new(b, d, t=self.tt)
        self.gamma, self.Wh = gain(), rnd(vocab, d, std=0.1)
        self.labels = torch.randint(0, vocab, (b,), device="cuda", generator=gen)
        self.mask = (torch.arange(b, device="cuda") % seq >= seq // 4).to(torch.uint8)
        self.labels[self.mask == 0] = -1
        self.off = torch.arange(batch + 1, device="cuda") * seq
        self.head = B.make_head_desc(b, d, vocab, code)
        self.logp, self.lse, self.dlogp, self.loss = new(b), new(b), new(b), new(1)
        self.ref = -6 + 0.3 * torch.randn(b, device="cuda", generator=gen)
        self.old = -6 + 0.3 * torch.randn(b, device="cuda", generator=gen)
        self.adv = torch.randn(batch, device="cuda", generator=gen)
        self.dWh, self.dgamma, self.dtop = new(vocab, d), new(d), new(b, d, t=self.tt)
        self.pref = B.make_preference_desc(b, batch // 2, 0.1)
        self.pol = B.make_policy_desc(b, batch, 0.2, 0.28, 0.05, B.MEAN_SEQUENCES)
        self.ws = {k: Guarded(n) for k, n in dict(
            stack=B.mecefo_stack_ckpt_workspace_bytes(self.desc, self.attn, r, r, r), fwd=B.mecefo_head_workspace_bytes(self.head, False),
            bwd=B.mecefo_head_workspace_bytes(self.head, True), pref=B.mecefo_preference_workspace_bytes(self.pref),
            pol=B.mecefo_policy_workspace_bytes(self.pol)).items()}

    def run(self, stream=None):
        w = {k: g.ws for k, g in self.ws.items()}
        B.mecefo_stack_fwd_neighbor_ckpt(self.desc, self.attn, self.lw, self.X0, self.H, self.X, w["stack"], stream)
        B.mecefo_head_logprob_fwd(self.head, self.X, self.gamma, self.Wh, self.labels, self.logp, self.lse, w["fwd"], stream)
        if self.loss_kind == "preference":
            B.mecefo_preference_loss(self.pref, self.logp, self.ref, self.mask, self.off, self.loss, None, None, self.dlogp, w["pref"], stream)
        else:
            B.mecefo_policy_loss(self.pol, self.logp, self.old, self.ref, self.adv, self.mask, self.off, self.loss, None, None,
                                 self.dlogp, w["pol"], stream)
        B.mecefo_head_logprob_bwd(self.head, self.X, self.gamma, self.Wh, self.labels, self.lse, self.dlogp, self.dtop, self.dgamma,
                                  self.dWh, 0, w["bwd"], stream)
        B.mecefo_stack_bwd_skip_ckpt(self.desc, self.lw, self.H, self.lr, B.SIDE_INPUT, self.dtop, self.dX, 0, w["stack"], stream)

    def results(self):
        return dict(X=self.X, logp=self.logp, lse=self.lse, loss=self.loss, dlogp=self.dlogp, dtop=self.dtop, dgamma=self.dgamma,
                    dWh=self.dWh, dX=self.dX, **{f"{k}{i}": t for i, q in enumerate(self.low) for k, t in q.items() if k[0] == "d"},
                    **{f"q{i}{j}": t for i, x in enumerate(self.q) for j, t in enumerate(x)})

    def copies(self):
        torch.cuda.synchronize()
        return {k: t.clone() for k, t in self.results().items()}


def h64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("loss", ["preference", "policy"])
def test_step_against_the_oracle_link_by_link(dtype, loss):
    s = Step(dtype, loss=loss)
    s.run()
    for k, g in s.ws.items():
        g.check(k)
    # each link from the values that the one before it handed over
    x = h64(s.X)
    rs = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + float(np.float32(1e-6)))
    N, gamma, Wh = x * rs, h64(s.gamma), h64(s.Wh)
    U = N * gamma
    gate = 2e-2 if dtype == "bf16" else 1e-5      # the gates of the block calls: several bf16 roundings in a row
    logp, lse = T.head_fwd(U, Wh, h64(s.labels).astype(int))
    assert relerr(h64(s.logp), logp) <= gate and relerr(h64(s.lse), lse) <= gate
    mask, off = s.mask.cpu().numpy(), s.off.cpu().numpy()
    if loss == "preference":
        want = T.preference(h64(s.logp), h64(s.ref), mask, off, float(np.float32(0.1)))
    else:
        want = T.policy(h64(s.logp), h64(s.old), h64(s.ref), h64(s.adv), mask, off, float(np.float32(0.2)), float(np.float32(0.28)),
                        float(np.float32(0.05)), True)
    assert relerr(h64(s.dlogp), want["dlogp"]) <= 1e-6 and abs(float(s.loss) - want["loss"]) <= 1e-5 * max(1, abs(want["loss"]))
    dU, dWh = T.head_bwd(U, Wh, h64(s.labels).astype(int), h64(s.dlogp))
    dN = dU * gamma
    assert relerr(h64(s.dWh), dWh) <= gate and relerr(h64(s.dgamma), (dU * N).sum(axis=0)) <= gate
    assert relerr(h64(s.dtop), rs * (dN - N * (dN * N).mean(axis=1, keepdims=True))) <= gate
    g = h64(s.dtop)
    for l in range(s.layers - 1, -1, -1):
        w, q = s.W[l], s.low[l]
        Hl = T.ckpt_unpack(s.q[l][0].cpu().numpy(), s.q[l][1].cpu().numpy(), s.d)
        o = O.block_bwd_skip(Hl, g, h64(w["g_ffn"]), h64(w["Wg"]), h64(w["Wu"]), h64(w["Wd"]), *[h64(p) for p in s.P[l]], 1e-6)
        for k in ("dWg", "dWu", "dWd"):
            assert relerr(h64(q[k]), o[k]) <= gate, (l, k)
        assert relerr(h64(q["dg_ffn"]), o["dgamma"]) <= gate
        g = o["dX"]
    assert relerr(h64(s.dX), g) <= 2 * gate      # two layers


@pytest.mark.parametrize("loss", ["preference", "policy"])
def test_step_replays_from_a_graph(loss):
    B.mecefo_init()
    s = Step(loss=loss)
    s.run()
    eager = s.copies()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.run(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for i in range(4):
        for t in s.results().values():
            t.fill_(1)
        for g in s.ws.values():
            g.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        got = s.copies()
        assert all(torch.equal(eager[k], got[k]) for k in eager), i
        s.X0.mul_(1.0)
        (s.X0.float() @ s.X0.float().t()).sum().item()      # the program's own work between the replays
    s.X0.mul_(0.5)      # the graph reads its inputs where they are
    s.run()
    eager = s.copies()
    graph.replay()
    got = s.copies()
    assert all(torch.equal(eager[k], got[k]) for k in eager)


def test_two_graphs_with_workspaces_of_their_own_may_overlap():
    B.mecefo_init()
    steps = [Step(loss=k) for k in ("preference", "policy")]
    eager = []
    for s in steps:
        s.run()
        eager.append(s.copies())
    graphs = []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(torch.cuda.current_stream())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        torch.cuda.synchronize()
        for s in steps:
            for t in s.results().values():
                t.fill_(1)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, e in zip(steps, eager):
            got = s.copies()
            assert all(torch.equal(e[k], got[k]) for k in e)


@pytest.mark.parametrize("b,d,v", [(1, 64, 7), (77, 128, 1001), (600, 64, 515)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ["all", "scored"])
def test_head_stays_inside_its_workspace(b, d, v, dtype, rows, mecefo_option):
    mecefo_option("head", rows)
    tt, code = (torch.bfloat16, B.BF16) if dtype == "bf16" else (torch.float32, B.F32)
    X, W, gamma = (torch.randn(s, device="cuda").to(tt) for s in ((b, d), (v, d), (d,)))
    labels, logp, lse = torch.randint(0, v, (b,), device="cuda"), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    desc = B.make_head_desc(b, d, v, code)
    for g in (None, gamma):
        fwd, bwd = (Guarded(B.mecefo_head_workspace_bytes(desc, k)) for k in (False, True))
        B.mecefo_head_logprob_fwd(desc, X, g, W, labels, logp, lse, fwd.ws)
        fwd.check("forward")
        B.mecefo_head_logprob_bwd(desc, X, g, W, labels, lse, logp, torch.empty_like(X), None if g is None else torch.empty(d, device="cuda"),
                                  torch.empty(v, d, device="cuda"), 0, bwd.ws)
        bwd.check("backward")
