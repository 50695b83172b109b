"""What a call writes must not lie over what it reads: refused on the host, before anything is enqueued."""
import pytest

from paper_2510_16415_amd import binding as B
from tests.test_operators_host import INV, STREAM, at, refused

TOKENS, SEQS = 40, 4
PREFERENCE = dict(logp=4 * TOKENS, ref_logp=4 * TOKENS, mask=TOKENS, offsets=8 * (SEQS + 1), loss=4, margins=2 * SEQS, rewards=4 * SEQS,
                  dlogp=4 * TOKENS)
POLICY = dict(logp=4 * TOKENS, old_logp=4 * TOKENS, ref_logp=4 * TOKENS, advantage=4 * SEQS, mask=TOKENS, offsets=8 * (SEQS + 1), loss=4,
              kl=4, clipped=4, dlogp=4 * TOKENS)
WRITTEN = ("loss", "margins", "rewards", "kl", "clipped", "dlogp")


def pairs(spans):
    return [(w, o) for w in spans if w in WRITTEN for o in spans if o != w]


def overlaps(call, desc, spans, need, moved):
    """The arrays 512 bytes apart, `moved` elsewhere; the workspace behind them."""
    a = {n: 512 * (i + 1) for i, n in enumerate(spans)}
    a.update(ws=16384)
    a.update(moved)
    refused(INV, "overlaps", call, desc, *[at(a[n]) for n in spans], at(a["ws"])[:need], STREAM)


@pytest.mark.parametrize("written,other", pairs(PREFERENCE))
def test_preference(written, other):
    d = B.make_preference_desc(TOKENS, SEQS // 2)
    need, lo = B.mecefo_preference_workspace_bytes(d), 512 * (1 + list(PREFERENCE).index(other))
    for place in (lo, (lo + PREFERENCE[other] - 1) // 4 * 4):      # the first bytes of the other one, and its last
        overlaps(B.mecefo_preference_loss, d, PREFERENCE, need, {written: place})


@pytest.mark.parametrize("written,other", pairs(POLICY))
def test_policy(written, other):
    d = B.make_policy_desc(TOKENS, SEQS, kl_coef=0.1)
    need, lo = B.mecefo_policy_workspace_bytes(d), 512 * (1 + list(POLICY).index(other))
    for place in (lo, (lo + POLICY[other] - 1) // 4 * 4):
        overlaps(B.mecefo_policy_loss, d, POLICY, need, {written: place})


def test_an_advantage_per_token_is_as_long_as_the_tokens():
    d = B.make_policy_desc(TOKENS, SEQS, advantage_per_token=True)
    at_adv = 512 * (1 + list(POLICY).index("advantage"))
    overlaps(B.mecefo_policy_loss, d, POLICY, B.mecefo_policy_workspace_bytes(d), dict(loss=at_adv + 4 * TOKENS - 4))


@pytest.mark.parametrize("name", list(POLICY))
def test_the_losses_workspaces(name):
    d = B.make_policy_desc(TOKENS, SEQS, kl_coef=0.1)
    need = B.mecefo_policy_workspace_bytes(d)
    overlaps(B.mecefo_policy_loss, d, POLICY, need, {name: 16384 + (need - 8) // 8 * 8})
    if name in PREFERENCE:
        d = B.make_preference_desc(TOKENS, SEQS // 2)
        need = B.mecefo_preference_workspace_bytes(d)
        overlaps(B.mecefo_preference_loss, d, PREFERENCE, need, {name: 16384})


def kept(q=None, e=None, cols=32):
    """A checkpoint of 2 rows, far from the other arguments where nothing else is said."""
    g = -(-cols // 32)
    base = at().data_ptr()
    return B.Ckpt(base + (q if q is not None else 57344 + 1024 * g), base + (e if e is not None else 61440 + 64 * g), 32 * g + 16, g + 1)


BLOCK = B.make_desc(2, 32, 64, B.BF16, ld_act_d=40)
DX, WS = 12288, 32768      # dX: 2 rows of stride 40, 144 bytes from the first element to the last


def block(**k):
    need = B.mecefo_block_ckpt_workspace_bytes(BLOCK)
    a = dict(desc=BLOCK, H=kept(), dOut=at(512), gamma=at(1024), Wg=at(2048), Wu=at(2048), Wd=at(2048), Pg=None, Pu=None, Pd=None,
             side=B.SIDE_INPUT, dX=at(DX), dgamma=at(14336), dWg=at(16384), dWu=at(20480), dWd=at(28672), accumulate=0,
             ws=at(WS)[:need], G=None, Z=None, exact_wgrad_mask=7, stream=STREAM)
    a.update(k)
    assert WS + need < 57344
    return a


@pytest.mark.parametrize("place", [DX, DX + 128, DX - 48])
@pytest.mark.parametrize("name", ["H", "G", "Z"])
def test_dx_over_a_checkpoint(name, place):
    cols = 32 if name == "H" else 64
    both = {} if name == "H" else dict(G=kept(cols=64), Z=kept(cols=64, q=60160, e=63488))
    both[name] = kept(cols=cols, q=place)
    refused(INV, f"dX overlaps checkpoint {name}", B.mecefo_block_bwd_skip_ckpt, **block(**both))
    both[name] = kept(cols=cols, e=place + 14 if place == DX + 128 else max(place, DX - 1))
    refused(INV, f"dX overlaps checkpoint {name}", B.mecefo_block_bwd_skip_ckpt, **block(**both))


@pytest.mark.parametrize("name", ["H", "G", "Z"])
def test_a_workspace_over_a_checkpoint(name):
    need = B.mecefo_block_ckpt_workspace_bytes(BLOCK) - 256      # the rest is for the alignment of the base
    for place in (WS, WS + need - 16):
        both = {} if name == "H" else dict(G=kept(cols=64), Z=kept(cols=64, q=60160, e=63488))
        both[name] = kept(cols=32 if name == "H" else 64, q=place)
        refused(INV, f"the workspace overlaps checkpoint {name}", B.mecefo_block_bwd_skip_ckpt, **block(**both))


def test_stacks_over_the_checkpoints_of_any_layer():
    d, a = B.make_desc(2, 32, 64, B.BF16), B.make_attn_desc(1, 2, 1, 32)
    need = B.mecefo_stack_ckpt_workspace_bytes(d, a)
    assert WS + need < 57344
    layers, low, ws = B.layer_weights([{}, {}]), (B.LayerLowrank * 2)(), at(WS)[:need]
    for bad, text in ((kept(q=512), "overlaps checkpoint H"), (kept(e=512 + 127), "overlaps checkpoint H"), (kept(q=WS + 1024), "the workspace overlaps")):
        for ks in ([bad, kept(q=60000 // 16 * 16)], [kept(q=60000 // 16 * 16), bad]):
            ks = B.ckpt_array(ks)
            refused(INV, text, B.mecefo_stack_fwd_neighbor_ckpt, d, a, layers, at(), ks, at(512), ws, STREAM)
            refused(INV, text, B.mecefo_stack_bwd_skip_ckpt, d, layers, ks, low, B.SIDE_INPUT, at(), at(512), 0, ws, STREAM)
