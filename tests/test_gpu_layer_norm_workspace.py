"""Gradients of the layer norm without those of weight and bias need no workspace."""
import pytest
import torch

import paper_2408_11746_amd as mst

gpu = pytest.mark.gpu
FAKE = 0x10000


def test_no_rows_and_no_sums():
    shape = mst.LayerNormShape(0, 64, 1e-5, mst.MST_F32, mst.MST_F32, mst.MST_F32)
    mst.mst_layer_norm_bwd(shape, None, None, None, None, None, None, None, None, None, None, None, stream=0)


@pytest.mark.parametrize("dweight,dbias", [(FAKE, None), (None, FAKE), (FAKE, FAKE)])
def test_sums_need_one(dweight, dbias):
    shape = mst.LayerNormShape(4, 64, 1e-5, mst.MST_F32, mst.MST_F32, mst.MST_F32)
    with pytest.raises(mst.MstError) as e:
        mst.mst_layer_norm_bwd(shape, FAKE, None, None, None, FAKE, None, FAKE, dweight, dbias, None, None, stream=0)
    assert e.value.code == -1


@gpu
@pytest.mark.parametrize("width", [64, 1001, 5000])
def test_the_same_gradient(width):
    from attention_util import DEV, space
    gen = torch.Generator(device=DEV).manual_seed(width)
    s, dy = (torch.randn(37, width, generator=gen, device=DEV) for _ in range(2))
    w = torch.randn(width, generator=gen, device=DEV)
    shape = mst.LayerNormShape(37, width, 1e-5, mst.MST_F32, mst.MST_F32, mst.MST_F32)
    one, both = torch.empty_like(s), torch.empty_like(s)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    mst.mst_layer_norm_bwd(shape, s, None, w, None, dy, None, one, None, None, None, None)
    mst.mst_layer_norm_bwd(shape, s, None, w, None, dy, None, both, dw, db, None, space(mst.mst_layer_norm_workspace_bytes(shape)))
    torch.cuda.synchronize()
    assert torch.equal(one, both)
