"""Workspaces of norm and loss lie on the GPU that the call runs on, one byte behind the other: others are refused before anything is launched.  (No GPU: these pointers are never read.)"""
import pytest
import torch

import paper_2408_11746_amd as mst

FAKE = 0x10000
NORM, LOSS = mst.LayerNormShape(4, 64, 1e-5, 0, 0, 0), mst.VocabLossShape(4, 64, 100, 1)
CALLS = [lambda ws: mst.mst_layer_norm_bwd(NORM, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ws, stream=0),
         lambda ws: mst.mst_vocab_loss_fwd(LOSS, FAKE, FAKE, FAKE, FAKE, FAKE, ws, stream=0),
         lambda ws: mst.mst_vocab_loss_bwd(LOSS, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ws, stream=0)]


# (few bytes: the library refuses them too, so that nothing is launched where the binding does not)
@pytest.mark.parametrize("call", CALLS, ids=["norm", "loss", "loss_bwd"])
@pytest.mark.parametrize("ws", [torch.empty(16, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8).expand(16)], ids=["host", "one byte"])
def test_refused(call, ws):
    with pytest.raises(ValueError, match="workspace"):
        call(ws)


@pytest.mark.parametrize("call", CALLS, ids=["norm", "loss", "loss_bwd"])
def test_none(call):
    with pytest.raises(mst.MstError):
        call(None)
