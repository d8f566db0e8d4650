"""What a row does not see has no part in its results, whatever the row, the keys or their product hold: padded queries that are no
numbers, and products that overflow in a block that only other rows of the same tile selected."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
from attention_util import tensor  # noqa: E402
from test_gpu_block_attention import Run, _check, _selection  # noqa: E402


def _padded(dtype, D, H, G, block):
    rng = np.random.default_rng(D + H)
    B, T, n_select = 3, 150, 3
    lengths = [150, 77, 5]
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, T, H, D)), dtype)
    k, v = tensor(rng.standard_normal((B, T, G, D)), dtype), tensor(rng.standard_normal((B, T, G, D)), dtype)
    blocks = _selection(rng, B, G, T, block, n_select, lengths)
    bad_q, bad_d = q.clone(), d_o.clone()
    for b, n in enumerate(lengths):
        bad_q[b, :T - n], bad_d[b, :T - n] = float("nan"), float("nan")
        bad_q[b, :T - n:3], bad_d[b, :T - n:3] = float("inf"), -float("inf")
    return lengths, blocks, q, k, v, d_o, bad_q, bad_d


PADDED = [(64, 2, 1, 32), (64, 3, 1, 64), (128, 2, 2, 64), (40, 4, 1, 128), (128, 2, 1, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,block", PADDED)
def test_padded_queries_may_hold_anything(D, H, G, block, dtype):
    lengths, blocks, q, k, v, d_o, bad_q, bad_d = _padded(dtype, D, H, G, block)
    clean, run = Run(q, k, v, blocks, block, 0.2, dtype, lengths), Run(bad_q, k, v, blocks, block, 0.2, dtype, lengths)
    few = Run(bad_q, k, v, blocks, block, 0.2, dtype, lengths, decode=True)
    assert torch.equal(run.o, clean.o) and torch.equal(run.lse, clean.lse)
    for b, n in enumerate(lengths):
        for x in (run, few):
            assert (x.o[b, :q.shape[1] - n] == 0).all() and torch.isneginf(x.lse[b, :, :q.shape[1] - n]).all()


def _overflow(dtype, D, R, block, signs):
    """Odd rows do not read block 0, whose products with them are beyond fp32 (or, of two signs, no number); even rows read it."""
    rng = np.random.default_rng(R + D)
    B, T, G, n_select = 1, 3 * block + 5, 2, 3
    H = R * G
    q, d_o = rng.standard_normal((B, T, H, D)), rng.standard_normal((B, T, H, D))
    k, v = rng.standard_normal((B, T, G, D)), rng.standard_normal((B, T, G, D))
    odd = np.arange(T) % 2 == 1
    blocks = np.full((B, G, T, n_select), -1, dtype=np.int32)
    for t in range(T):
        own = t // block
        row = sorted(({0} if not odd[t] else set()) | {min(1, own), own}) if own > 0 else ([-1] if odd[t] else [0])
        blocks[:, :, t, :len(row)] = row
    k[..., :2], q[..., :2], v[..., :2], d_o[..., :2] = 0, 0, 0, 0
    for c, sign in enumerate(signs):
        k[:, :block, :, c], v[:, :block, :, c] = sign * 2.0 ** 80, sign * 2.0 ** 80
        q[:, odd, :, c], d_o[:, odd, :, c] = 2.0 ** 60, 2.0 ** 60
    return (tensor(q, dtype), tensor(k, dtype), tensor(v, dtype), tensor(d_o, dtype)), blocks, [T]


OVERFLOWS = [(64, 1, 32), (64, 3, 64), (128, 2, 64), (96, 1, 128)]


@pytest.mark.parametrize("signs", [(1,), (-1,), (1, -1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R,block", OVERFLOWS)
def test_products_that_overflow_where_a_row_does_not_look(D, R, block, dtype, signs):
    (q, k, v, d_o), blocks, lengths = _overflow(dtype, D, R, block, signs)
    _check(Run(q, k, v, blocks, block, 0.3, dtype), q, k, v, blocks, block, 0.3, dtype, lengths)
    _check(Run(q, k, v, blocks, block, 0.3, dtype, decode=True), q, k, v, blocks, block, 0.3, dtype, lengths)


def test_a_row_that_is_no_number_stays_one():
    # of the row that holds it: its own results, and nothing of its neighbours'
    rng = np.random.default_rng(3)
    B, T, H, G, D, block = 1, 100, 2, 1, 64, 32
    q, k, v = (tensor(rng.standard_normal((B, T, n, D)), "bf16") for n in (H, G, G))
    blocks = _selection(rng, B, G, T, block, 2, [T])
    clean = Run(q, k, v, blocks, block, 0.05, "bf16")
    q[0, 50, 1, 3] = float("nan")
    run = Run(q, k, v, blocks, block, 0.05, "bf16")
    assert run.o[0, 50, 1].isnan().all() and run.lse[0, 1, 50].isnan()
    same = torch.ones(T, H, dtype=torch.bool, device=q.device)
    same[50, 1] = False
    assert torch.equal(run.o[0][same], clean.o[0][same]) and torch.equal(run.lse[0].T[same], clean.lse[0].T[same])
