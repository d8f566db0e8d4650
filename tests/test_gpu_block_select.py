"""Summaries of key blocks and the selection by their scores: whole numbers, equal to the oracle's."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import attention as oat

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, lengths_of, tensor, wide  # noqa: E402


def _shape(B, T, S, H, G, D, block, n_select, dtype, lengths=None):
    return mst.BlockAttentionShape(B, T, S, H, G, D, block, n_select, 0.5, TYPES[dtype][0], None if lengths is None else lengths_of(lengths))


def _summaries(shape, k, block, new_tokens, sums=None, scales=None):
    B, S, G, D = k.shape
    nb = -(-S // block)
    if sums is None:
        sums = torch.full((B, G, nb, D), 99, dtype=torch.int8, device=DEV)
        scales = torch.full((B, G, nb), -1.0, device=DEV)
    mst.mst_key_summary(shape, k, sums, scales, new_tokens)
    torch.cuda.synchronize()
    return sums, scales


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (8, "bf16"), (80, "f32"), (40, "bf16"), (128, "f32")])
def test_summaries(block, D, dtype):
    rng = np.random.default_rng(block + D)
    B, S, G = 2, 3 * block + 5, 3
    lengths = [S, 2 * block - 1]
    k = rng.standard_normal((B, S, G, D)) * np.exp(3 * rng.standard_normal((B, 1, G, 1)))
    k[0, :block, 0] = 0                                             # a block of zeros
    k[0, block:2 * block, 1] = 1e30 if dtype == "f32" else 2.0 ** 100
    k[0, 2 * block:3 * block, 2] = 2.0 ** -120                      # below the least unit
    k = tensor(k, dtype)
    shape = _shape(B, S, S, G, G, D, block, 4, dtype, lengths)
    sums, scales = _summaries(shape, k, block, S)
    ref = oat.key_summary(wide(k), block, lengths)
    nb = -(-S // block)
    for b in range(B):
        for g in range(G):
            for j in range(nb):
                if (b, g, j) in ref:
                    assert np.array_equal(sums[b, g, j].cpu().numpy(), ref[b, g, j][0]), (b, g, j)
                    assert float(scales[b, g, j]) == ref[b, g, j][1]
                else:                                               # incomplete blocks stay as they are
                    assert (sums[b, g, j] == 99).all() and float(scales[b, g, j]) == -1


@pytest.mark.parametrize("new_tokens", [1, 3, 31, 32, 33, 200])
def test_summaries_of_what_new_tokens_completed(new_tokens):
    rng = np.random.default_rng(new_tokens)
    B, S, G, D, block = 4, 160, 2, 16, 32
    k = tensor(rng.standard_normal((B, S, G, D)), "bf16")
    lengths = [160, 128, 97, 20]
    shape = _shape(B, new_tokens, S, G, G, D, block, 4, "bf16", lengths)
    whole, whole_scales = _summaries(shape, k, block, S)
    sums, scales = _summaries(shape, k, block, new_tokens)
    for b, n in enumerate(lengths):
        for j in range(5):
            done = (j + 1) * block <= n and (j + 1) * block > n - new_tokens
            assert torch.equal(sums[b, :, j], whole[b, :, j]) if done else bool((sums[b, :, j] == 99).all()), (b, j)
            assert torch.equal(scales[b, :, j], whole_scales[b, :, j]) if done else bool((scales[b, :, j] == -1).all())


@pytest.mark.parametrize("B,T,S,H,G,D,block,n_select,dtype,lengths", [
    (1, 200, 200, 2, 2, 64, 32, 4, "bf16", None),
    (2, 150, 150, 6, 2, 40, 32, 3, "f32", [150, 77]),               # left-padded: rows before the first key
    (2, 70, 300, 4, 1, 128, 64, 2, "bf16", [300, 190]),             # a piece of a prompt
    (3, 1, 515, 8, 2, 64, 32, 8, "bf16", [515, 32, 1]),             # single tokens
    (2, 5, 260, 40, 2, 16, 32, 4, "bf16", [260, 3]),                # fewer keys than queries; twenty heads to a key head
    (1, 40, 64, 1, 1, 8, 32, 1, "bf16", None),                      # the own block alone
    (2, 33, 96, 2, 1, 24, 32, 64, "f32", [96, 0]),                  # more than there are; a sequence without keys
    (1, 65, 9000, 1, 1, 16, 32, 12, "bf16", None),                  # more blocks than stay in registers
    (1, 3, 40000, 1, 1, 16, 32, 20, "bf16", None),
    (1, 17, 700, 1, 1, 16, 32, 20, "bf16", None),
    (1, 20, 2100, 1, 1, 16, 32, 40, "bf16", None),
])
def test_selection(B, T, S, H, G, D, block, n_select, dtype, lengths):
    rng = np.random.default_rng(T + S)
    n = lengths or [S] * B
    q, k = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, S, G, D)), dtype)
    shape = _shape(B, T, S, H, G, D, block, n_select, dtype, lengths)
    sums, scales = _summaries(shape, k, block, S)
    got = torch.full((B, G, T, n_select), -7, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, q, sums, scales, got)
    torch.cuda.synchronize()
    ref = oat.select(wide(q), sums.cpu().numpy(), scales.cpu().numpy(), block, n_select, n, G)
    np.testing.assert_array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("T", [3, 100])
@pytest.mark.parametrize("blocks,n_select", [(100, 6), (300, 33), (1500, 64)])
def test_ties_and_zeros(T, blocks, n_select):
    rng = np.random.default_rng(T + blocks)
    block, D = 32, 16
    S = blocks * block
    sums = np.repeat(rng.integers(-2, 3, (1, 1, blocks, 1)), D, axis=3).astype(np.int8)
    scales = np.full((1, 1, blocks), 0.25, dtype=np.float32)
    q = np.ones((1, T, 1, D)) * np.where(rng.random((1, T, 1, 1)) < 0.2, 0.0, 1.0)      # a zero query ties all blocks
    shape = _shape(1, T, S, 1, 1, D, block, n_select, "f32")
    got = torch.empty(1, 1, T, n_select, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, tensor(q, "f32"), torch.from_numpy(sums).to(DEV), torch.from_numpy(scales).to(DEV), got)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(got.cpu().numpy(), oat.select(q, sums, scales, block, n_select, [S], 1))


def test_a_single_token_selects_what_the_prompt_selected():
    rng = np.random.default_rng(3)
    B, S, H, G, D, block, n_select = 2, 400, 6, 2, 64, 32, 5
    q, k = tensor(rng.standard_normal((B, S, H, D)), "bf16"), tensor(rng.standard_normal((B, S, G, D)), "bf16")
    shape = _shape(B, S, S, H, G, D, block, n_select, "bf16")
    sums, scales = _summaries(shape, k, block, S)
    all_ = torch.empty(B, G, S, n_select, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, q, sums, scales, all_)
    for t in (0, 31, 32, 255, 399):
        one = _shape(B, 1, S, H, G, D, block, n_select, "bf16", [t + 1] * B)
        got = torch.empty(B, G, 1, n_select, dtype=torch.int32, device=DEV)
        mst.mst_block_select(one, q[:, t:t + 1], sums, scales, got)
        torch.cuda.synchronize()
        assert torch.equal(got[:, :, 0], all_[:, :, t]), t


def test_what_is_not_finite_still_selects_blocks_of_the_sequence():
    B, S, H, G, D, block, n_select = 1, 320, 2, 1, 16, 32, 4
    q, k = torch.randn(B, S, H, D, device=DEV), torch.randn(B, S, G, D, device=DEV)
    q[0, ::3, 0, 0] = float("nan")
    q[0, 1::3, 1, 2] = float("inf")
    k[0, ::50] = float("-inf")
    k[0, 7] = float("nan")
    shape = _shape(B, S, S, H, G, D, block, n_select, "f32")
    sums, scales = _summaries(shape, k, block, S)
    got = torch.empty(B, G, S, n_select, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, q, sums, scales, got)
    torch.cuda.synchronize()
    rows = got.cpu().numpy()[0, 0]
    for t, row in enumerate(rows):
        own, kept = t // block, [j for j in row if j >= 0]
        assert kept == sorted(set(kept)) and kept[-1] == own and len(kept) == min(n_select, own + 1) and (row[len(kept):] == -1).all()


CASES_OF_MANY = [
    (1, 1100, 1100, 2, 2, 64, 32, 4, "bf16", None),
    (2, 650, 650, 6, 2, 40, 32, 3, "f32", [650, 77]),               # left-padded
    (9, 70, 300, 8, 2, 128, 64, 2, "bf16", [300, 190] * 4 + [70]),
    (200, 1, 515, 24, 6, 64, 32, 8, "bf16", [515, 32, 1, 0] * 50),  # many single tokens
    (13, 41, 260, 40, 2, 16, 32, 4, "bf16", [260, 3, 41] * 4 + [0]),  # twenty heads to a key head
    (5, 257, 300, 1, 1, 8, 32, 1, "bf16", None),                    # the own block alone
    (8, 129, 160, 2, 1, 24, 32, 64, "f32", [96, 0] * 4),            # more than there are
    (16, 65, 9000, 1, 1, 16, 32, 12, "bf16", None),                 # more blocks than stay in registers
    (70, 17, 700, 1, 1, 16, 32, 20, "bf16", None),
    (1, 1031, 2100, 2, 1, 104, 32, 40, "f32", None),
]


@pytest.mark.parametrize("B,T,S,H,G,D,block,n_select,dtype,lengths", CASES_OF_MANY)
def test_selection_of_many_queries(B, T, S, H, G, D, block, n_select, dtype, lengths):
    assert B * T * G >= 1024                                        # (fewer go another way)
    test_selection(B, T, S, H, G, D, block, n_select, dtype, lengths)


@pytest.mark.parametrize("blocks,n_select", [(100, 6), (300, 33), (1500, 64)])
def test_ties_and_zeros_of_many_queries(blocks, n_select):
    test_ties_and_zeros(1100, blocks, n_select)


def test_few_and_many_queries_agree():
    # the last queries of long sequences: all at once, and a few at a time
    rng = np.random.default_rng(17)
    B, T, S, H, G, D, block, n_select = 4, 300, 5000, 4, 2, 72, 32, 10
    q, k = tensor(rng.standard_normal((B, T, H, D)), "bf16"), tensor(rng.standard_normal((B, S, G, D)), "bf16")
    lengths = [S, 301, 299, 4000]
    shape = _shape(B, T, S, H, G, D, block, n_select, "bf16", lengths)
    sums, scales = _summaries(shape, k, block, S)
    many = torch.empty(B, G, T, n_select, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, q, sums, scales, many)
    for t0 in range(0, T, 100):
        part = _shape(B, 100, S, H, G, D, block, n_select, "bf16", [n - T + t0 + 100 for n in lengths])
        few = torch.empty(B, G, 100, n_select, dtype=torch.int32, device=DEV)
        mst.mst_block_select(part, q[:, t0:t0 + 100], sums, scales, few)
        torch.cuda.synchronize()
        assert torch.equal(few, many[:, :, t0:t0 + 100])


def test_what_is_not_finite_among_many_queries():
    B, S, H, G, D, block, n_select = 4, 320, 2, 1, 16, 32, 4
    q, k = torch.randn(B, S, H, D, device=DEV), torch.randn(B, S, G, D, device=DEV)
    q[0, ::3, 0, 0] = float("nan")
    q[1, 1::3, 1, 2] = float("inf")
    k[2, ::50] = float("-inf")
    k[3, 7] = float("nan")
    shape = _shape(B, S, S, H, G, D, block, n_select, "f32")
    sums, scales = _summaries(shape, k, block, S)
    got = torch.empty(B, G, S, n_select, dtype=torch.int32, device=DEV)
    mst.mst_block_select(shape, q, sums, scales, got)
    torch.cuda.synchronize()
    for b in range(B):
        for t, row in enumerate(got.cpu().numpy()[b, 0]):
            own, kept = t // block, [j for j in row if j >= 0]
            assert kept == sorted(set(kept)) and kept[-1] == own and len(kept) == min(n_select, own + 1) and (row[len(kept):] == -1).all()
