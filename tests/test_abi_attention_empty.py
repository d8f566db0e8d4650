"""Calls of the attention over selected blocks that have nothing to write take null buffers, as the header says; no GPU is met."""
import ctypes as C

import pytest

import paper_2408_11746_amd as mst
from test_abi_attention import FAKE, _attn, _view

EMPTY = C.byref(mst.HeadsView(0, 0, 0, 0))


@pytest.mark.parametrize("kw", [dict(batch=0), dict(queries=0), dict(queries=0, keys=0)])
def test_calls_for_no_queries(kw):
    s, L = _attn(**kw), mst.lib()
    assert L.mst_block_select(s._ref, EMPTY, None, None, None, None) == 0
    assert L.mst_block_plan(s._ref, None, None, 0, None) == 0
    assert L.mst_block_attention_fwd(s._ref, *[EMPTY] * 3, None, EMPTY, None, None, 0, None) == 0
    assert L.mst_block_attention_decode(s._ref, *[EMPTY] * 3, None, EMPTY, None, None) == 0


@pytest.mark.parametrize("kw", [dict(batch=0), dict(queries=0, keys=0)])
def test_gradients_of_nothing(kw):
    assert mst.lib().mst_block_attention_bwd(_attn(**kw)._ref, *[EMPTY] * 3, None, EMPTY, None, *[EMPTY] * 4, None, 0, None) == 0


@pytest.mark.parametrize("kw,new", [(dict(batch=0), 100), (dict(keys=0), 100), (dict(keys=31), 100), (dict(), 0)])
def test_summaries_of_no_complete_block(kw, new):
    assert mst.lib().mst_key_summary(_attn(**kw)._ref, EMPTY, None, None, new, None) == 0


def test_what_is_written_is_still_asked_for():
    s, L, v = _attn(), mst.lib(), C.byref(_view())
    assert L.mst_key_summary(s._ref, v, None, FAKE, 1, None) == -1 and L.mst_key_summary(s._ref, v, FAKE, None, 1, None) == -1
    assert L.mst_key_summary(s._ref, EMPTY, FAKE, FAKE, 1, None) == -1
    assert L.mst_block_plan(s._ref, FAKE, None, 1 << 30, None) == -1
    none = _attn(queries=0)                                        # gradients of 100 keys that nobody reads: zeros, and a workspace
    assert L.mst_block_attention_bwd(none._ref, EMPTY, v, v, None, EMPTY, None, EMPTY, EMPTY, v, v, None, 1 << 30, None) == -1
    assert L.mst_block_attention_bwd(none._ref, EMPTY, v, v, None, EMPTY, None, EMPTY, EMPTY, EMPTY, v, FAKE, 1 << 30, None) == -1
    assert L.mst_block_attention_bwd(none._ref, EMPTY, v, v, None, EMPTY, None, EMPTY, EMPTY, v, v, FAKE, 1, None) == -3
