"""The loss over vocabularies that are worked on in several pieces: sums taken up again, labels and results of later pieces, last pieces that are shorter, or too short for all ranges of a sum.
Against float64, with the bounds of test_gpu_vocab_loss.py.

That there are several is read off the workspace, which holds what one piece needs for every column: dz of the rows (padded to 256; three parts in fp32) in the backward pass, and the parts of the
embedding's rows (padded to 64 columns) where it is not read as it is."""
import pytest
import torch

import paper_2408_11746_amd as mst

pytestmark = pytest.mark.gpu
from test_gpu_vocab_loss import Case  # noqa: E402


def _padded(n, to):
    return -(-n // to) * to


def _pieces_at_least(c, backward):
    wide, rows = _padded(c.W, 64), _padded(c.T, 256)
    split = c.dtype == "f32" or wide != c.W
    column = (6 if c.dtype == "f32" else 2) * ((rows if backward else 0) + (wide if split else 0))
    return -(-column * _padded(c.V, 256) // mst.mst_vocab_loss_workspace_bytes(c.shape, backward))


@pytest.mark.parametrize("dtype,tokens,width,vocab,pieces", [
    # (sums of dh by tiles of 128 x 128 where the width is 64, by those of 256 x 256 where it is more; logits by either)
    ("bf16", 2048, 64, 200000, 2), ("bf16", 4096, 64, 140000, 3), ("bf16", 1500, 512, 200003, 2),
    ("f32", 2048, 64, 100000, 3), ("f32", 1500, 512, 60000, 2), ("f32", 1024, 768, 100003, 3),
])
def test_gradients(dtype, tokens, width, vocab, pieces):
    c = Case(31, tokens, width, vocab, dtype, unlabelled=0.1, uniform=True)
    assert _pieces_at_least(c, True) >= pieces
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype,tokens,width,vocab", [("f32", 100, 2048, 50001), ("f32", 700, 2048, 100001), ("bf16", 70, 2040, 140000), ("bf16", 700, 2040, 140000)])
def test_losses(dtype, tokens, width, vocab):
    """(with the workspace of the forward alone; 100 and 70 tokens by tiles of 128 x 128, 700 by those of 256 x 256)"""
    c = Case(32, tokens, width, vocab, dtype)
    assert _pieces_at_least(c, False) >= 2
    c.ws = c.ws[:mst.mst_vocab_loss_workspace_bytes(c.shape, False) + 64]
    c.ws[-64:] = 99
    c.forward()
    c.check(dh=False, dE=False)


def test_a_last_piece_with_fewer_ranges():
    """eleven pieces of 2816 columns at most, of which the last has 60: one step of a sum that the others split in two"""
    c = Case(33, 30000, 64, 28220, "f32", unlabelled=0.1)
    rows, wide, piece, splits = 30208, 64, 2816, 2
    # dz and the embedding of a piece, the states, the sums (columns padded to 256), and less than 1 MB of numbers per row: with other pieces or ranges this test needs other sizes
    known = 6 * (rows + wide) * piece + 6 * rows * wide + 4 * splits * rows * 256
    assert known <= mst.mst_vocab_loss_workspace_bytes(c.shape, True) < known + (1 << 20)
    c.forward()
    c.backward()
    c.check()
    torch.cuda.empty_cache()
