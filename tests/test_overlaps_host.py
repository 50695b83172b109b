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
