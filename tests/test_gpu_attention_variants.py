"""Every code that the sizes of a call choose, against the oracle: block sizes with each padded width, several items to a block, signs
of the scale in either type, widths of the single-token form, and the gradients of many norms."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import attention as oat

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, space, tensor, wide  # noqa: E402
from test_gpu_block_attention import Run, _check, _selection  # noqa: E402
from test_gpu_qk_norm import _case, _on  # noqa: E402


def _inputs(rng, B, T, S, H, G, D, dtype):
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, T, H, D)), dtype)
    return q, tensor(rng.standard_normal((B, S, G, D)) + rng.standard_normal((1, 1, G, D)), dtype), tensor(rng.standard_normal((B, S, G, D)), dtype), d_o


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,S,H,G,D,block,n_select,lengths", [
    (1, 150, 150, 2, 1, 128, 32, 3, None),                          # short blocks of wide heads
    (1, 140, 140, 4, 2, 80, 32, 3, None),
    (2, 75, 200, 3, 1, 104, 32, 4, [200, 60]),
    (1, 300, 300, 2, 1, 64, 128, 2, None),                          # long blocks of narrow heads
    (1, 300, 300, 2, 2, 40, 128, 2, None),
    (2, 90, 310, 2, 1, 56, 128, 3, [310, 50]),
    (1, 300, 300, 2, 1, 128, 64, 2, None),                          # two heads of a workgroup in the single-token form
    (1, 20, 300, 2, 1, 96, 32, 4, None),                            # few rows for the card: one head and eight wavefronts there
    (1, 7, 300, 1, 1, 64, 64, 4, None),
])
def test_sizes(B, T, S, H, G, D, block, n_select, lengths, dtype):
    rng = np.random.default_rng(T + S + D)
    n = lengths or [S] * B
    q, k, v, d_o = _inputs(rng, B, T, S, H, G, D, dtype)
    blocks = _selection(rng, B, G, T, block, n_select, n)
    run = Run(q, k, v, blocks, block, D ** -0.5, dtype, lengths, d_o)
    _check(run, q, k, v, blocks, block, D ** -0.5, dtype, n, d_o)
    _check(Run(q, k, v, blocks, block, D ** -0.5, dtype, lengths, decode=True), q, k, v, blocks, block, D ** -0.5, dtype, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [32, 64, 128])
def test_blocks_that_many_rows_read(block, D, dtype):
    # more rows than one workgroup of dK and dV takes (512): partial sums, joined
    rng = np.random.default_rng(block + D)
    B, T, H, G = 1, 2 * block + 90, 8, 1
    q, k, v, d_o = _inputs(rng, B, T, T, H, G, D, dtype)
    blocks = np.full((B, G, T, 3), -1, dtype=np.int32)
    for t in range(T):
        row = sorted({0, min(1, t // block), t // block})
        blocks[0, 0, t, :len(row)] = row
    assert T * H > 2 * 512
    run = Run(q, k, v, blocks, block, D ** -0.5, dtype, None, d_o)
    _check(run, q, k, v, blocks, block, D ** -0.5, dtype, [T], d_o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [48, 128])
@pytest.mark.parametrize("scale", [-0.3, 0.0, -1e-30])
def test_signs_of_the_scale(scale, D, dtype):
    rng = np.random.default_rng(D)
    B, T, H, G, block = 1, 140, 4, 2, 64
    q, k, v, d_o = _inputs(rng, B, T, T, H, G, D, dtype)
    blocks = _selection(rng, B, G, T, block, 2, [T])
    _check(Run(q, k, v, blocks, block, scale, dtype, None, d_o), q, k, v, blocks, block, scale, dtype, [T], d_o)
    _check(Run(q, k, v, blocks, block, scale, dtype, decode=True), q, k, v, blocks, block, scale, dtype, [T])


@pytest.mark.parametrize("H,G", [(8, 3), (6, 0), (0, 5)])
@pytest.mark.parametrize("D,interleaved,x,y", [(256, False, "f32", "bf16"), (64, True, "bf16", "bf16")])
def test_gradients_of_more_norms_than_workgroups(D, interleaved, x, y, H, G):
    # the backward keeps to 1024 workgroups, shared between queries and keys, that take their vectors in turn
    B, T, eps = 2, 2500 if D == 256 else 9000, 1e-6
    rng, rows, (wq, wk), table, positions = _case(D + H, B, T, H, G, D, D, x)
    rows = rows[:, :, :H + G]
    shape = mst.QKNormShape(B, T, H, G, D, D, interleaved, table.shape[0], eps, TYPES[x][0], TYPES[y][0])
    per = 256 // (32 if D == 256 else 8)
    assert B * T * (-(-H // 2) + -(-G // 2)) > 1024 * per
    dy = tensor(rng.standard_normal((B, T, H + G, D)), y)
    dx = torch.full_like(rows, float("nan"))
    dwq, dwk = torch.full((D,), float("nan"), device=DEV), torch.full((D,), float("nan"), device=DEV)
    mst.mst_qk_norm_rotate_bwd(shape, rows[:, :, :H], rows[:, :, H:], _on(wq), _on(wk), _on(table), _on(positions), dy[:, :, :H], dy[:, :, H:],
                               dx[:, :, :H], dx[:, :, H:], dwq if H else None, dwk if G else None, space(mst.mst_qk_norm_rotate_workspace_bytes(shape)))
    torch.cuda.synchronize()
    cos, sin = np.split(table.astype(np.float64)[positions], 2, axis=-1)
    u = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[x]
    for n, w, h, dw in ((H, wq, slice(0, H), dwq), (G, wk, slice(H, H + G), dwk)):
        if n == 0:
            continue
        xs, w, d = wide(rows[:, :, h]), w.astype(np.float64), wide(dy[:, :, h])
        rx, rw = oat.norm_rotate_bwd(xs, w, cos, sin, D, interleaved, eps, d)
        # as in the tests of few norms: sums of D products and two dozen operations in fp32, then the output's rounding
        r = 1 / np.sqrt((xs * xs).mean(-1, keepdims=True) + eps)
        dmax = 2 * np.abs(d).max(-1, keepdims=True)
        size = r * np.abs(w).max() * (dmax + np.abs(xs) * r * dmax)
        assert (np.abs(wide(dx[:, :, h]) - rx) <= (2 * D + 24) * 2.0 ** -24 * size + 2 * u * np.abs(rx)).all()
        total = (np.abs(xs) * r * dmax).sum((0, 1, 2))
        # a thread's own sum, then sums over the lanes and rows: far fewer terms in a row than vectors
        assert (np.abs(wide(dw) - rw) <= (D + B * T * n) * 2.0 ** -24 * total).all()
        # ... and what a lost or doubled workgroup of vectors would do is far above what is seen
        assert np.linalg.norm(wide(dw) - rw) <= 1e-4 * np.linalg.norm(rw)
