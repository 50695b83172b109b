"""What the head, loss and checkpoint calls refuse, on the host, before anything is enqueued."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2510_16415_amd import binding as B

BIG = torch.zeros(1 << 16, dtype=torch.uint8)      # host memory: no refused call may touch it


def at(offset=0):
    return BIG[(-BIG.data_ptr()) % 256 + offset:]


def refused(status, text, fn, *a, **k):
    with pytest.raises(B.MecefoError) as e:
        fn(*a, **k)
    assert e.value.status == status and text in str(e.value), str(e.value)


INV, UNS, WS = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE_TOO_SMALL
STREAM = 0


def raw_ckpt(q=256, e=8192, ld_q=64, ld_e=2):
    base = at().data_ptr()
    return B.Ckpt(base + q if q is not None else None, base + e if e is not None else None, ld_q, ld_e)


@pytest.mark.parametrize("change,status,text", [
    (dict(k=None), INV, "ckpt is NULL"),
    (dict(k=raw_ckpt(q=None)), INV, "required"),
    (dict(k=raw_ckpt(e=None)), INV, "required"),
    (dict(k=raw_ckpt(q=264)), INV, "16-byte"),
    (dict(k=raw_ckpt(ld_q=72)), INV, "multiple of 16"),
    (dict(k=raw_ckpt(ld_q=48)), INV, "ld_q >= 64"),
    (dict(k=raw_ckpt(ld_e=1)), INV, "ld_e >= 2"),
    (dict(k=raw_ckpt(ld_q=1 << 31)), UNS, "2 GiB"),
    (dict(k=raw_ckpt(ld_e=1 << 31)), UNS, "2 GiB"),
    (dict(k=raw_ckpt(q=16384 + 16)), INV, "overlap"),
    (dict(k=raw_ckpt(e=300)), INV, "overlap"),
    (dict(dtype=2), INV, "dtype"),
    (dict(rows=-1), INV, "rows >= 0"),
    (dict(cols=0), INV, "cols >= 1"),
    (dict(ldx=32), INV, "row stride"),
    (dict(ldx=44), INV, "multiple of 8"),
    (dict(x=8), INV, "16-byte"),
    (dict(x=None), INV, "X is NULL"),
    (dict(rows=1 << 30), UNS, "2 GiB"),
])
def test_checkpoint_refusals(change, status, text):
    a = dict(dtype=B.BF16, x=16384, rows=3, cols=40, ldx=48, k=raw_ckpt())
    a.update(change)
    X = None if a["x"] is None else at(a["x"])
    refused(status, text, B.mecefo_checkpoint_pack, a["dtype"], X, a["rows"], a["cols"], a["ldx"], a["k"], STREAM)
    refused(status, text, B.mecefo_checkpoint_unpack, a["dtype"], a["k"], a["rows"], a["cols"], X, a["ldx"], STREAM)


def test_checkpoints_of_no_rows_are_nothing_to_do():
    B.mecefo_checkpoint_pack(B.BF16, None, 0, 40, 48, raw_ckpt(q=None, e=None), STREAM)
    B.mecefo_checkpoint_unpack(B.F32, raw_ckpt(q=None, e=None), 0, 40, None, 40, STREAM)


def head(**k):
    a = dict(tokens=4, d_model=16, vocab=10, dtype=B.BF16, grad_dtype=B.F32)
    a.update(k)
    return B.make_head_desc(**a)


@pytest.mark.parametrize("desc,status,text", [
    (dict(dtype=3), INV, "dtype"),
    (dict(dtype=B.F32, grad_dtype=B.BF16), UNS, "grad_dtype"),
    (dict(tokens=-1), INV, "tokens >= 0"),
    (dict(d_model=0, ld_act_d=8, ld_w=8), INV, "d_model >= 1"),
    (dict(vocab=0), INV, "vocab >= 1"),
    (dict(ld_act_d=8), INV, "row stride"),
    (dict(ld_w=8), INV, "row stride"),
    (dict(d_model=12), UNS, "multiple of 8"),
    (dict(ld_w=20), INV, "multiple of 8"),
    (dict(logit_scale=float("inf")), INV, "logit_scale"),
    (dict(logit_scale=float("nan")), INV, "logit_scale"),
    (dict(tokens=1 << 27), UNS, "2 GiB"),
    (dict(vocab=1 << 30), UNS, "2 GiB"),
])
def test_head_descriptor_refusals(desc, status, text):
    refused(status, text, B.mecefo_head_workspace_bytes, head(**desc), True)
    refused(status, text, B.mecefo_head_logprob_fwd, head(**desc), at(), None, at(), at(), at(), at(), at(), STREAM)


@pytest.mark.parametrize("dtype,tokens,d_model,vocab,forward,backward", [
    (B.BF16, 16384, 64, 65536, True, False),          # dz of 2 GiB
    (B.BF16, 16384, 64, 65528, True, True),
    (B.BF16, 131072, 64, 65536, False, False),        # the forward's parts too
    (B.BF16, 131071, 64, 65536, True, False),
    (B.F32, 16384, 64, 32768, False, False),
    (B.F32, 16384, 64, 32760, True, True),
    (B.BF16, 64, 4096, 262143, True, True),           # W below 2 GiB, an fp32 dW above
    (B.BF16, 64, 4096, 262144, False, False),
    (B.F32, 64, 4096, 131071, True, True),
    (B.F32, 64, 4096, 131072, False, False),
])
def test_head_sizes_at_their_limits(dtype, tokens, d_model, vocab, forward, backward):
    h = head(dtype=dtype, tokens=tokens, d_model=d_model, vocab=vocab)
    for back, allowed in ((False, forward), (True, backward)):
        if allowed:
            assert B.mecefo_head_workspace_bytes(h, back) > 0
        else:
            refused(UNS, "2 GiB", B.mecefo_head_workspace_bytes, h, back)


def head_args(h, **change):
    """Places for every argument of the backward, apart from each other."""
    a = dict(X=at(256), gamma=at(1024), W=at(2048), labels=at(2976), lse=at(3200), dlogp=at(3300), dX=at(3584),
             dgamma=at(4096), dW=at(5120), ws=at(8192))
    a.update(change)
    return a


@pytest.mark.parametrize("change,status,text", [
    (dict(X=None), INV, "X is NULL"), (dict(W=None), INV, "W is NULL"), (dict(labels=None), INV, "labels is NULL"),
    (dict(X=at(264)), INV, "X is not 16-byte"), (dict(gamma=at(1028)), INV, "gamma is not"), (dict(W=at(2056)), INV, "W is not"),
    (dict(labels=at(2980)), INV, "labels is not 8-byte"), (dict(lse=at(3201)), INV, "lse is not 4-byte"),
    (dict(ws=None), WS, "needed"), (dict(ws=at(8192)[:64]), WS, "needed"),
])
def test_head_pointer_refusals(change, status, text):
    h = head()
    a = head_args(h, **change)
    refused(status, text, B.mecefo_head_logprob_fwd, h, a["X"], a["gamma"], a["W"], a["labels"], at(6144), a["lse"], a["ws"], STREAM)
    refused(status, text, B.mecefo_head_logprob_bwd, h, a["X"], a["gamma"], a["W"], a["labels"], a["lse"], a["dlogp"], a["dX"],
            a["dgamma"], a["dW"], 0, a["ws"], STREAM)


@pytest.mark.parametrize("change,text", [
    (dict(lse=None), "lse is NULL"), (dict(dlogp=None), "dlogp is NULL"), (dict(dX=None), "dX is NULL"), (dict(dW=None), "dW is NULL"),
    (dict(gamma=None), "dgamma requested"), (dict(dX=at(256)), "dX overlaps X"), (dict(dX=at(272)), "dX overlaps X"),
    (dict(dW=at(2048)), "dW overlaps W"), (dict(dW=at(256)), "dW overlaps X"), (dict(dX=at(2064)), "dX overlaps W"),
    (dict(dX=at(5136)), "dW overlaps dX"), (dict(dlogp=at(3302)), "dlogp is not"), (dict(dgamma=at(4100)), "dgamma is not"),
])
def test_head_backward_refusals(change, text):
    h = head()
    a = head_args(h, **change)
    refused(INV, text, B.mecefo_head_logprob_bwd, h, a["X"], a["gamma"], a["W"], a["labels"], a["lse"], a["dlogp"], a["dX"],
            a["dgamma"], a["dW"], 0, a["ws"], STREAM)


def test_head_forward_needs_logp():
    a = head_args(head())
    refused(INV, "logp is NULL", B.mecefo_head_logprob_fwd, head(), a["X"], None, a["W"], a["labels"], None, None, a["ws"], STREAM)


def test_head_of_no_tokens_is_nothing_to_do():
    B.mecefo_head_logprob_fwd(head(tokens=0), None, None, at(), None, None, None, at(8192), STREAM)


@pytest.mark.parametrize("desc,status,text", [
    (dict(tokens=-1), INV, ">= 0"), (dict(pairs=-1), INV, ">= 0"), (dict(tokens=1 << 29), UNS, "2 GiB"),
    (dict(pairs=(1 << 19) + 1), UNS, "2^20"), (dict(pairs=(1 << 31) - 1), UNS, "2^20"), (dict(beta=float("nan")), INV, "finite"), (dict(margin=float("inf")), INV, "finite"),
    (dict(grad_scale=float("inf")), INV, "finite"), (dict(label_smoothing=-0.1), INV, "label_smoothing"),
    (dict(label_smoothing=1.5), INV, "label_smoothing"), (dict(label_smoothing=float("nan")), INV, "label_smoothing"),
])
def test_preference_descriptor_refusals(desc, status, text):
    d = B.make_preference_desc(**{**dict(tokens=10, pairs=2), **desc})
    refused(status, text, B.mecefo_preference_workspace_bytes, d)
    refused(status, text, B.mecefo_preference_loss, d, at(), at(), at(), at(), at(), at(), at(), at(), at(), STREAM)


@pytest.mark.parametrize("desc,status,text", [
    (dict(tokens=-1), INV, ">= 0"), (dict(sequences=-1), INV, ">= 0"), (dict(tokens=1 << 29), UNS, "2 GiB"),
    (dict(sequences=(1 << 20) + 1), UNS, "2^20"), (dict(clip_low=-0.1), INV, "clip_low"), (dict(clip_low=1.1), INV, "clip_low"),
    (dict(clip_high=-0.1), INV, "clip_high"), (dict(clip_high=float("inf")), INV, "clip_high"),
    (dict(kl_coef=float("nan")), INV, "kl_coef"), (dict(grad_scale=float("nan")), INV, "grad_scale"), (dict(mean=2), INV, "mean"),
])
def test_policy_descriptor_refusals(desc, status, text):
    d = B.make_policy_desc(**{**dict(tokens=10, sequences=2), **desc})
    refused(status, text, B.mecefo_policy_workspace_bytes, d)
    refused(status, text, B.mecefo_policy_loss, d, at(), at(), at(), at(), at(), at(), at(), at(), at(), at(), at(), STREAM)


def test_loss_pointer_refusals():
    d = B.make_preference_desc(10, 2)
    names = ["logp", "ref_logp", "mask", "offsets", "loss", "margins", "rewards", "dlogp"]
    good = {n: at(256 * (i + 1)) for i, n in enumerate(names)}
    for n in ("logp", "offsets", "loss", "dlogp"):
        refused(INV, f"{n} is NULL", B.mecefo_preference_loss, d, *{**good, n: None}.values(), at(4096), STREAM)
    for n in ("logp", "ref_logp", "offsets", "loss", "margins", "rewards", "dlogp"):
        refused(INV, f"{n} is not", B.mecefo_preference_loss, d, *{**good, n: at(2)}.values(), at(4096), STREAM)
    refused(WS, "needed", B.mecefo_preference_loss, d, *good.values(), at(4096)[:16], STREAM)
    refused(WS, "needed", B.mecefo_preference_loss, d, *good.values(), None, STREAM)
    d = B.make_policy_desc(10, 2, kl_coef=0.1)
    names = ["logp", "old_logp", "ref_logp", "advantage", "mask", "offsets", "loss", "kl", "clipped", "dlogp"]
    good = {n: at(256 * (i + 1)) for i, n in enumerate(names)}
    for n in ("logp", "old_logp", "advantage", "offsets", "loss", "dlogp"):
        refused(INV, f"{n} is NULL", B.mecefo_policy_loss, d, *{**good, n: None}.values(), at(4096), STREAM)
    for n in ("logp", "old_logp", "ref_logp", "advantage", "offsets", "loss", "kl", "clipped", "dlogp"):
        refused(INV, f"{n} is not", B.mecefo_policy_loss, d, *{**good, n: at(2)}.values(), at(4096), STREAM)
    refused(INV, "kl_coef needs", B.mecefo_policy_loss, d, *{**good, "ref_logp": None}.values(), at(4096), STREAM)
    refused(WS, "needed", B.mecefo_policy_loss, d, *good.values(), at(4096)[:16], STREAM)


def block_args(**k):
    a = dict(desc=B.make_desc(2, 32, 64, B.BF16), H=raw_ckpt(), dOut=at(512), gamma=at(1024), Wg=at(2048), Wu=at(2048), Wd=at(2048),
             Pg=None, Pu=None, Pd=None, side=B.SIDE_INPUT, dX=at(12288), dgamma=at(14336), dWg=at(20480), dWu=at(24576), dWd=at(28672),
             accumulate=0, ws=BIG, G=None, Z=None, exact_wgrad_mask=7, stream=STREAM)
    a.update(k)
    return a


@pytest.mark.parametrize("change,status,text", [
    (dict(H=None), INV, "checkpoint H is NULL"), (dict(H=raw_ckpt(ld_q=16)), INV, "checkpoint H"),
    (dict(G=raw_ckpt()), INV, "G and Z must both"), (dict(Z=raw_ckpt()), INV, "G and Z must both"),
    (dict(G=raw_ckpt(ld_q=32), Z=raw_ckpt()), INV, "checkpoint G"), (dict(G=raw_ckpt(), Z=raw_ckpt(ld_e=1)), INV, "checkpoint Z"),
    (dict(exact_wgrad_mask=8), INV, "exact_wgrad_mask"), (dict(exact_wgrad_mask=3), INV, "projection Pd is NULL"),
    (dict(dX=at(528)), INV, "dX overlaps dOut"), (dict(gamma=None), INV, "dgamma requested"), (dict(ws=BIG[:512]), WS, "needed"),
])
def test_block_backward_from_checkpoints_refusals(change, status, text):
    refused(status, text, B.mecefo_block_bwd_skip_ckpt, **block_args(**change))


def test_block_workspace_has_room_for_what_is_unpacked():
    d = B.make_desc(100, 64, 200, B.BF16)
    more = B.mecefo_block_ckpt_workspace_bytes(d, 8, 8, 8) - B.mecefo_workspace_bytes(d, 8, 8, 8)
    assert more >= 100 * 2 * 64


def test_stack_with_checkpoints_refusals():
    d, a = B.make_desc(4, 32, 64, B.BF16), B.make_attn_desc(1, 4, 1, 32)
    layers = B.layer_weights([{}, {}])
    ks = B.ckpt_array([raw_ckpt(), raw_ckpt(ld_q=16)])
    refused(INV, "checkpoint H", B.mecefo_stack_fwd_neighbor_ckpt, d, a, layers, at(), ks, at(512), BIG, STREAM)
    refused(INV, "checkpoint H", B.mecefo_stack_bwd_skip_ckpt, d, layers, ks, (B.LayerLowrank * 2)(), B.SIDE_INPUT, at(), at(512), 0, BIG, STREAM)
    good = B.ckpt_array([raw_ckpt()])
    refused(INV, "1 entries in H, 2 layers", B.mecefo_stack_fwd_neighbor_ckpt, d, a, layers, at(), good, at(512), BIG, STREAM)
    refused(INV, "1 entries in H", B.mecefo_stack_bwd_skip_ckpt, d, layers, good, (B.LayerLowrank * 2)(), B.SIDE_INPUT, at(), at(512), 0, BIG, STREAM)
    refused(INV, "3 entries in lowrank", B.mecefo_stack_bwd_skip_ckpt, d, layers, ks, (B.LayerLowrank * 3)(), B.SIDE_INPUT, at(), at(512), 0, BIG, STREAM)
    refused(INV, "required", B.mecefo_stack_fwd_neighbor_ckpt, d, a, layers, at(), None, at(512), BIG, STREAM)
    refused(INV, "required", B.mecefo_stack_bwd_skip_ckpt, d, layers, None, (B.LayerLowrank * 2)(), B.SIDE_INPUT, at(), at(512), 0, BIG, STREAM)
    assert B.mecefo_stack_ckpt_workspace_bytes(d, a, 4, 4, 4) >= B.mecefo_block_ckpt_workspace_bytes(d, 4, 4, 4)


def test_descriptors_have_the_layout_of_the_header():
    assert C.sizeof(B.Ckpt) == 32 and C.sizeof(B.HeadDesc) == 48 and C.sizeof(B.PreferenceDesc) == 32 and C.sizeof(B.PolicyDesc) == 40


def test_ranges_of_sequences_and_slices(tmp_path):
    here = os.path.dirname(os.path.abspath(__file__))
    exe = tmp_path / "loss_ranges"
    subprocess.run(["g++", "-std=c++17", "-Wall", os.path.join(here, "loss_ranges.cpp"), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout == "ok\n"


def test_head_option():
    refused(INV, "option head", B.mecefo_set_option, "head", "some")
    h = head(tokens=4096, d_model=1024, vocab=32000)
    narrow = head(tokens=131072, d_model=512, vocab=1000)      # as many operations, dW too small for a list to pay
    need, small = {}, {}
    try:
        for v in ("all", "scored", "auto"):
            B.mecefo_set_option("head", v)
            small[v] = B.mecefo_head_workspace_bytes(narrow, True)
            need[v] = B.mecefo_head_workspace_bytes(h, True), B.mecefo_head_workspace_bytes(head(), True), B.mecefo_head_workspace_bytes(h, False)
    finally:
        B.mecefo_set_option("head", "auto")
    assert need["auto"][0] == need["scored"][0] >= need["all"][0] + 4096 * (1024 * 2 + 20) and need["auto"][1] == need["all"][1] < need["scored"][1]
    assert len({n[2] for n in need.values()}) == 1 and small["auto"] == small["all"] < small["scored"]
