"""Scores below everything that fp32 holds, of finite heads: they weigh nothing, first block or last, and a row that has no others is a
row without keys."""
import numpy as np
import pytest
import torch

from oracle import attention as oat

pytestmark = pytest.mark.gpu
from attention_util import assert_within, bounds, tensor, wide  # noqa: E402
from test_gpu_block_attention import Run  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [0, 1])
@pytest.mark.parametrize("D,R,block", [(64, 1, 32), (64, 3, 64), (128, 2, 64), (96, 1, 128)])
def test_lowest_scores(D, R, block, low, dtype):
    rng = np.random.default_rng(D + R)
    B, T, G = 1, 3 * block + 5, 2
    H, scale = R * G, 0.3
    q, d_o = rng.standard_normal((B, T, H, D)), rng.standard_normal((B, T, H, D))
    k, v = rng.standard_normal((B, T, G, D)), rng.standard_normal((B, T, G, D))
    odd = (np.arange(T) % 2 == 1) & (np.arange(T) >= 2 * block)
    blocks = np.full((B, G, T, 3), -1, dtype=np.int32)
    for t in range(T):
        row = sorted({0, min(1, t // block), t // block})
        blocks[:, :, t, :len(row)] = row
    none = T - 2                                                    # (odd) reads the low block alone
    assert odd[none]
    blocks[:, :, none] = [low, -1, -1]
    k[..., 0], q[..., 0] = 0, 0
    k[:, low * block:(low + 1) * block, :, 0] = -2.0 ** 80          # with the odd rows: -2^140
    q[:, odd, :, 0] = 2.0 ** 60
    q, k, v, d_o = (tensor(x, dtype) for x in (q, k, v, d_o))
    left = blocks.copy()                                            # what weighs anything
    for t in np.nonzero(odd)[0]:
        rest = [j for j in blocks[0, 0, t] if j != low and j >= 0]
        left[:, :, t] = rest + [-1] * (3 - len(rest))
    seen = oat.visible(left, block, [T], T, T)
    o, lse, grads, size, most = oat.attention(wide(q), wide(k), wide(v), seen, scale, wide(d_o))
    run = Run(q, k, v, blocks, block, scale, dtype, None, d_o)
    few = Run(q, k, v, blocks, block, scale, dtype, decode=True)
    n = D + int(seen.sum(-1).max())
    for x in (run, few):
        assert_within(wide(x.o), o, bounds(o, size["o"], "o", dtype, n, most), "o")
        got, full = wide(x.lse), ~np.isneginf(lse)
        assert np.isneginf(got[~full]).all() and (np.abs(got[full] - lse[full]) <= 2.0 ** -22 * (most + n + np.abs(lse[full]) + 4)).all()
        assert (x.o[0, none] == 0).all() and torch.isneginf(x.lse[0, :, none]).all()
    rows = int(seen.sum(2).max()) * R
    for name, g, got in zip(("dq", "dk", "dv"), grads, (run.dq, run.dk, run.dv)):
        assert_within(wide(got), g, bounds(g, size[name], name, dtype, n + D if name == "dq" else rows + 2 * D + n, most), name)
