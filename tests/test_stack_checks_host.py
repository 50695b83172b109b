"""A stack call that one of its layers makes impossible enqueues nothing: the layers are checked before the first one runs."""
import ctypes

import pytest

from paper_2510_16415_amd import binding as B
from tests.test_operators_host import BIG, INV, STREAM, WS, at, refused

DESC, ATTN = B.make_desc(2, 32, 64, B.BF16), B.make_attn_desc(1, 2, 1, 32)
N = 3


def layers(bad=None, **change):
    all_ = []
    for l in range(N):
        w = {k: at(2048 + 64 * i) for i, k in enumerate(("g_attn", "g_ffn", "Wq", "Wk", "Wv", "Wo", "Wg", "Wu", "Wd"))}
        if l == bad:
            w.update(change)
        all_.append(w)
    return B.layer_weights(all_)


def lowrank(bad=None, **change):
    arr = (B.LayerLowrank * N)()
    for l, a in enumerate(arr):
        for k in ("Pg", "Pu", "Pd"):
            setattr(a, k, B.Proj(at(4096).data_ptr(), 8, 8))
        for k in ("dg_ffn", "dWg", "dWu", "dWd"):
            setattr(a, k, at(8192).data_ptr())
        if l == bad:
            for k, v in change.items():
                setattr(a, k, v)
    return arr


def ckpts():
    return B.ckpt_array([B.Ckpt(at(1024).data_ptr(), at(1280).data_ptr(), 32, 1) for _ in range(N)])


def ws(need):
    assert 16384 + need < BIG.numel() - 512
    return at(16384)[:need]


FORWARD = [(dict(Wd=None), "Wd is NULL"), (dict(g_attn=None), "g_attn is NULL"), (dict(Wq=at(2056)), "Wq is not 16-byte")]


@pytest.mark.parametrize("bad", [1, N - 1])
@pytest.mark.parametrize("change,text", FORWARD)
def test_forward(change, text, bad):
    w = layers(bad, **change)
    H = [at(12288)] * N
    refused(INV, text, B.mecefo_stack_fwd_neighbor, DESC, ATTN, w, at(256), H, at(512), ws(B.mecefo_stack_workspace_bytes(DESC, ATTN)), STREAM)
    refused(INV, text, B.mecefo_stack_fwd_neighbor_ckpt, DESC, ATTN, w, at(256), ckpts(), at(512),
            ws(B.mecefo_stack_ckpt_workspace_bytes(DESC, ATTN)), STREAM)


BACKWARD = [(dict(), dict(dWd=None), "dWg, dWu, dWd are required"), (dict(Wg=None), dict(), "Wg is NULL"),
            (dict(), dict(Pu=B.Proj(None, 8, 8)), "projection Pu is NULL"), (dict(), dict(Pd=B.Proj(1 << 20, 65, 72)), "projection Pd: rank 65"),
            (dict(g_ffn=None), dict(), "dgamma requested")]


@pytest.mark.parametrize("bad", [0, 1])
@pytest.mark.parametrize("weights,low,text", BACKWARD)
def test_backward(weights, low, text, bad):
    w, q = layers(bad, **weights), lowrank(bad, **low)
    refused(INV, text, B.mecefo_stack_bwd_skip, DESC, w, [at(12288)] * N, q, B.SIDE_INPUT, at(256), at(512), 0,
            ws(B.mecefo_workspace_bytes(DESC, 8, 8, 8)), STREAM)
    refused(INV, text, B.mecefo_stack_bwd_skip_ckpt, DESC, w, ckpts(), q, B.SIDE_INPUT, at(256), at(512), 0,
            ws(B.mecefo_block_ckpt_workspace_bytes(DESC, 8, 8, 8)), STREAM)


def test_a_layer_whose_rank_needs_more_workspace():
    q = lowrank(0, Pd=B.Proj(at(4096).data_ptr(), 64, 64))
    need = B.mecefo_workspace_bytes(DESC, 8, 8, 8)
    refused(WS, "needed", B.mecefo_stack_bwd_skip, DESC, layers(), [at(12288)] * N, q, B.SIDE_INPUT, at(256), at(512), 0, ws(need), STREAM)
    need = B.mecefo_block_ckpt_workspace_bytes(DESC, 8, 8, 8)
    refused(WS, "needed", B.mecefo_stack_bwd_skip_ckpt, DESC, layers(), ckpts(), q, B.SIDE_INPUT, at(256), at(512), 0, ws(need), STREAM)


def mixed(modes, bad, change_in=None, change_out=None, q=None, policy=None, counters=None, need=None):
    inputs, grads = [], []
    for l in range(N):
        x = {k: at(2048 + 64 * i) for i, k in enumerate(("X", "H", "g_attn", "g_ffn", "Wq", "Wk", "Wv", "Wo", "Wg", "Wu", "Wd", "Q", "K", "V", "O", "L"))}
        g = {k: at(12288) for k in ("dg_attn", "dg_ffn", "dWq", "dWk", "dWv", "dWo", "dWg", "dWu", "dWd")}
        if l == bad:
            x.update(change_in or {})
            g.update(change_out or {})
        inputs.append(x)
        grads.append(g)
    need = need or B.mecefo_stack_mixed_workspace_bytes(DESC, ATTN, 8, 8, 8)
    return (DESC, ATTN, modes, inputs, grads, q or lowrank(), B.SIDE_INPUT, policy, counters, at(256), at(512), 0, ws(need), STREAM)


S, NB = B.MODE_STANDARD, B.MODE_NEIGHBOR


@pytest.mark.parametrize("modes,args,text", [
    ([S, S, NB], dict(bad=0, change_in=dict(Wo=None)), "Wo is NULL"), ([S, NB, S], dict(bad=0, change_out=dict(dWk=None)), "every gradient"),
    ([NB, S, S], dict(bad=0, change_in=dict(H=None)), "H is NULL"), ([NB, NB, S], dict(bad=1, q=lowrank(1, Pd=B.Proj(1 << 20, 65, 72))), "rank 65")])
def test_mixed_backward(modes, args, text):
    refused(INV, text, B.mecefo_stack_bwd_mixed, *mixed(modes, **args))


def test_mixed_backward_whose_refresh_needs_more_workspace():
    need = max(B.mecefo_block_full_workspace_bytes(DESC, ATTN), B.mecefo_workspace_bytes(DESC, 8, 8, 8))
    refresh = max(B.mecefo_projection_workspace_bytes(B.BF16, m, n, r) for m, n, r in ((64, 32, 8), (32, 64, 8)))
    assert need < refresh
    counters = (ctypes.c_int64 * N)(*[0] * N)
    refused(WS, "needed", B.mecefo_stack_bwd_mixed, *mixed([NB, NB, S], None, policy=B.RefreshPolicy(5, 1, 0, 1), counters=counters, need=need))
    assert list(counters) == [0] * N
