"""Tensors and checkpoints that lie close to each other: pieces of one buffer, each from its first element to its last."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as T
from paper_2510_16415_amd import binding as B
from tests.test_gpu_checkpoint import CODE, TYPE, values

pytestmark = pytest.mark.gpu


def up(n, a=256):
    return (n + a - 1) // a * a


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,wide", [(1, 64, 4096), (3, 40, 96), (50, 128, 512), (7, 33, 1024)])
def test_the_last_columns_of_a_wide_tensor(dtype, rows, cols, wide):
    """X is the last columns of a wider tensor, the checkpoint directly behind it, e within what q's last row leaves of its stride."""
    rng = np.random.default_rng([rows, cols, wide])
    tt, esz, g = TYPE[dtype], 2 if dtype == "bf16" else 4, -(-cols // 32)
    x = values(rng, rows, cols, dtype)
    first = (wide - cols) // 8 * 8
    at_q = up((rows * wide - (wide - first) + cols) * esz, 16)      # behind the last element of X
    ld_q, ld_e = 32 * g + 64, g + 5
    at_e = at_q + (rows - 1) * ld_q + 32 * g
    end = at_e + (rows - 1) * ld_e + g
    buf = torch.zeros(up(max(end, rows * wide * esz)), dtype=torch.uint8, device="cuda")
    X = buf[:rows * wide * esz].view(tt).view(rows, wide)[:, first:first + cols]
    X.copy_(torch.from_numpy(x))
    q = torch.as_strided(buf.view(torch.int8), (rows, 32 * g), (ld_q, 1), at_q)
    e = torch.as_strided(buf, (rows, g), (ld_e, 1), at_e)
    k = B.ckpt(q, e)
    B.mecefo_checkpoint_pack(CODE[dtype], X, rows, cols, wide, k)
    want_q, want_e = T.ckpt_pack(x)
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(e.cpu().numpy(), want_e)
    X.fill_(1.0)
    B.mecefo_checkpoint_unpack(CODE[dtype], k, rows, cols, X, wide)
    assert np.array_equal(X.float().cpu().numpy(), T.ckpt_unpack(want_q, want_e, cols))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(e.cpu().numpy(), want_e)
