"""Gradients of keys that no query reads: zeros, with no plan, outputs or log-sums to be given."""
import pytest
import torch

import paper_2408_11746_amd as mst

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, space  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block,D", [(32, 128), (64, 64), (128, 40)])
def test_no_queries(block, D, dtype):
    B, S, G = 2, 300, 3
    k, v = (torch.randn(B, S, G, D, device=DEV).to(TYPES[dtype][1]) for _ in range(2))
    dk, dv = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    shape = mst.BlockAttentionShape(B, 0, S, G, G, D, block, 4, 0.2, TYPES[dtype][0])
    none = mst.HeadsView(0, 0, 0, 0)
    ws = space(mst.mst_block_attention_workspace_bytes(shape, True))
    mst.mst_block_plan(shape, None, torch.empty(0, dtype=torch.uint8, device=DEV))
    mst.mst_block_attention_bwd(shape, none, k, v, None, none, None, none, none, dk, dv, ws)
    torch.cuda.synchronize()
    assert (dk == 0).all() and (dv == 0).all()
