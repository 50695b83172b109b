"""Limits of sizes and numbers: calls whose kernels take a wave per row refuse more rows than one launch has waves; the head refuses a
scale that is no number once it is turned to base 2."""
import pytest

from paper_2510_16415_amd import binding as B
from tests.test_operators_host import INV, STREAM, UNS, at, refused

MOST = (1 << 26) - 64


@pytest.mark.parametrize("dtype,d", [(B.BF16, 8), (B.F32, 4)])
def test_more_rows_than_waves(dtype, d):
    text = "2^26 - 64 tokens"
    h = B.make_head_desc(MOST + 1, d, 1, dtype)
    refused(UNS, text, B.mecefo_head_workspace_bytes, h, False)
    refused(UNS, text, B.mecefo_head_logprob_fwd, h, at(), None, at(), at(), at(), at(), at(), STREAM)
    f = B.make_desc(MOST + 1, d, d, dtype)
    refused(UNS, text, B.mecefo_block_bwd_skip_ex, f, at(), at(), at(), at(), at(), at(), None, None, None, B.SIDE_INPUT, at(512), None, at(), at(),
            at(), 0, at(), stream=STREAM)
    f, a = B.make_desc(1 << 26, d, d, dtype), B.make_attn_desc(8192, 8192, 1, d)
    refused(UNS, text, B.mecefo_block_fwd, f, a, {}, {}, at(), STREAM)
    refused(UNS, text, B.mecefo_block_bwd_full, f, a, {}, {}, 0, at(), STREAM)
    assert B.mecefo_head_workspace_bytes(B.make_head_desc(MOST, d, 1, dtype), False) > 0


@pytest.mark.parametrize("scale", [2.0 ** 127 * 1.001, -3.4e38])
def test_a_scale_beyond_base_2(scale):
    for dtype in (B.BF16, B.F32):
        refused(INV, "logit_scale", B.mecefo_head_workspace_bytes, B.make_head_desc(4, 8, 5, dtype, logit_scale=scale), False)
        assert B.mecefo_head_workspace_bytes(B.make_head_desc(4, 8, 5, dtype, logit_scale=-2.0 ** 127), True) > 0
