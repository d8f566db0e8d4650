"""What a row does not see has no part in its gradients: padded queries and gradients that are no numbers, and products that
overflow in a block that only other rows of the same tile selected."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
from attention_util import tensor  # noqa: E402
from test_gpu_attention_masked import OVERFLOWS, PADDED, _overflow, _padded  # noqa: E402
from test_gpu_block_attention import Run, _check, _selection  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,block", PADDED)
def test_padded_queries_and_their_gradients_may_hold_anything(D, H, G, block, dtype):
    lengths, blocks, q, k, v, d_o, bad_q, bad_d = _padded(dtype, D, H, G, block)
    clean, run = Run(q, k, v, blocks, block, 0.2, dtype, lengths, d_o), Run(bad_q, k, v, blocks, block, 0.2, dtype, lengths, bad_d)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(run, name), getattr(clean, name)), name
    for b, n in enumerate(lengths):
        assert (run.dq[b, :q.shape[1] - n] == 0).all()


@pytest.mark.parametrize("signs", [(1,), (-1,), (1, -1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R,block", OVERFLOWS)
def test_products_that_overflow_where_a_row_does_not_look(D, R, block, dtype, signs):
    (q, k, v, d_o), blocks, lengths = _overflow(dtype, D, R, block, signs)
    _check(Run(q, k, v, blocks, block, 0.3, dtype, None, d_o), q, k, v, blocks, block, 0.3, dtype, lengths, d_o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["q", "d_o"])
def test_a_row_that_is_no_number_stays_one(which, dtype):
    # of the queries' gradients the row's own is none, the others' are what they were
    rng = np.random.default_rng(4)
    B, T, H, G, D, block = 1, 100, 2, 1, 64, 32
    x = dict(zip(("q", "k", "v", "d_o"), (tensor(rng.standard_normal((B, T, n, D)), dtype) for n in (H, G, G, H))))
    blocks = _selection(rng, B, G, T, block, 2, [T])
    clean = Run(x["q"], x["k"], x["v"], blocks, block, 0.05, dtype, None, x["d_o"])
    x[which][0, 50, 1, 3] = float("nan")
    run = Run(x["q"], x["k"], x["v"], blocks, block, 0.05, dtype, None, x["d_o"])
    assert run.dq[0, 50, 1].isnan().all()
    same = torch.ones(T, H, dtype=torch.bool, device=run.dq.device)
    same[50, 1] = False
    assert torch.equal(run.dq[0][same], clean.dq[0][same])
