"""Refusals and sizes of the attention half that need no GPU: every argument is checked on the host, and these pointers are never read."""
import ctypes as C

import pytest

import paper_2408_11746_amd as mst

FAKE = 0x10000


def _view(token=64, head=64, data=FAKE, batch=6400):
    return mst.HeadsView(data, batch, token, head)


def _norm(**kw):
    a = dict(batch=1, tokens=4, heads=2, kv_heads=2, head_dim=64, rotated=64, interleaved=0, table_rows=8, eps=1e-6, in_type=0, out_type=0)
    a.update(kw)
    return mst.QKNormShape(*[a[n] for n, _ in mst.QKNormShape._fields_])


def _attn(**kw):
    a = dict(batch=1, queries=100, keys=100, heads=2, kv_heads=2, head_dim=64, block=32, n_select=4, scale=0.1, type=1, lengths=None)
    a.update(kw)
    return mst.BlockAttentionShape(**a)


@pytest.mark.parametrize("kw,code", [(dict(head_dim=60), -2), (dict(head_dim=264), -2), (dict(head_dim=0), -2), (dict(rotated=63), -2), (dict(rotated=66), -2),
                                     (dict(rotated=-2), -2), (dict(batch=-1), -2), (dict(tokens=-1), -2), (dict(heads=-1), -2), (dict(table_rows=0), -2),
                                     (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(in_type=2), -1), (dict(out_type=7), -1)])
def test_norm_refuses_shapes(kw, code):
    v, s = _view(), _norm(**kw)
    with pytest.raises(mst.MstError) as e:
        mst.mst_qk_norm_rotate(s, v, v, None, None, FAKE, None, v, v, stream=0)
    assert e.value.code == code
    assert mst.mst_qk_norm_rotate_workspace_bytes(s) == 0


def test_norm_refuses_arguments():
    v, s = _view(), _norm()
    bad = [_view(data=0), _view(data=FAKE + 8), _view(token=66), _view(token=-64), _view(head=2)]
    for x in bad:
        for args in ((x, v, FAKE, v, v), (v, x, FAKE, v, v), (v, v, FAKE, x, v), (v, v, FAKE, v, x)):
            with pytest.raises(mst.MstError) as e:
                mst.mst_qk_norm_rotate(s, args[0], args[1], None, None, args[2], None, args[3], args[4], stream=0)
            assert e.value.code == -1
    for table, weight in ((None, None), (FAKE + 4, None), (FAKE, FAKE + 4)):
        with pytest.raises(mst.MstError):
            mst.mst_qk_norm_rotate(s, v, v, weight, None, table, None, v, v, stream=0)
    with pytest.raises(mst.MstError):                               # an output may not be one vector for several
        mst.mst_qk_norm_rotate(s, v, v, None, None, FAKE, None, _view(token=0), v, stream=0)
    L = mst.lib()
    ref = C.byref
    need = mst.mst_qk_norm_rotate_workspace_bytes(s)
    assert need > 0
    for ws, n, code in ((None, need, -1), (FAKE, need - 1, -3)):
        assert L.mst_qk_norm_rotate_bwd(ref(s), ref(v), ref(v), None, None, FAKE, None, ref(v), ref(v), ref(v), ref(v), None, None, ws, n, None) == code
    assert L.mst_qk_norm_rotate(None, ref(v), ref(v), None, None, FAKE, None, ref(v), ref(v), None) == -1
    with pytest.raises(ValueError):
        import torch
        mst.heads(torch.zeros(2, 3, 64))
    with pytest.raises(ValueError):
        mst.heads(torch.zeros(2, 3, 64, 4).transpose(2, 3))


@pytest.mark.parametrize("kw,code", [(dict(head_dim=12), -2), (dict(head_dim=136), -2), (dict(block=16), -2), (dict(block=96), -2), (dict(n_select=0), -2),
                                     (dict(n_select=65), -2), (dict(heads=3), -2), (dict(heads=130, kv_heads=2), -2), (dict(kv_heads=0), -2), (dict(keys=-1), -2),
                                     (dict(keys=32 * 2048 + 1), -2), (dict(queries=-1), -2), (dict(batch=-1), -2), (dict(batch=40000), -2),
                                     (dict(queries=1 << 27), -2), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(type=2), -1),
                                     (dict(lengths=FAKE + 4), -1)])
def test_attention_refuses_shapes(kw, code):
    s, v = _attn(**kw), _view()
    assert mst.mst_block_plan_bytes(s) == 0 and mst.mst_block_attention_workspace_bytes(s, True) == 0 and mst.mst_block_attention_workspace_bytes(s, False) == 0
    calls = [lambda L: L.mst_key_summary(s._ref, C.byref(v), FAKE, FAKE, 1, None), lambda L: L.mst_block_select(s._ref, C.byref(v), FAKE, FAKE, FAKE, None),
             lambda L: L.mst_block_plan(s._ref, FAKE, FAKE, 1 << 40, None), lambda L: L.mst_block_attention_decode(s._ref, *[C.byref(v)] * 3, FAKE, C.byref(v), None, None),
             lambda L: L.mst_block_attention_fwd(s._ref, *[C.byref(v)] * 3, FAKE, C.byref(v), FAKE, FAKE, 1 << 40, None),
             lambda L: L.mst_block_attention_bwd(s._ref, *[C.byref(v)] * 3, FAKE, C.byref(v), FAKE, *[C.byref(v)] * 4, FAKE, 1 << 40, None)]
    for call in calls:
        assert call(mst.lib()) == code


def test_attention_refuses_arguments():
    s, v, L = _attn(), _view(), mst.lib()
    r = C.byref
    plan, ws = mst.mst_block_plan_bytes(s), mst.mst_block_attention_workspace_bytes(s, True)
    assert plan > 0 and ws >= mst.mst_block_attention_workspace_bytes(s, False) > 0
    assert L.mst_block_plan(s._ref, FAKE, FAKE, plan - 1, None) == -3 and L.mst_block_plan(s._ref, None, FAKE, plan, None) == -1
    assert L.mst_key_summary(s._ref, r(v), FAKE, FAKE, -1, None) == -1 and L.mst_key_summary(s._ref, r(v), FAKE + 1, FAKE, 1, None) == -1
    assert L.mst_block_select(s._ref, r(v), FAKE, FAKE, None, None) == -1
    good = [r(v)] * 3
    assert L.mst_block_attention_fwd(s._ref, *good, FAKE, r(v), None, FAKE, ws, None) == -1
    assert L.mst_block_attention_fwd(s._ref, *good, FAKE, r(v), FAKE, FAKE, 1, None) == -3
    assert L.mst_block_attention_bwd(s._ref, *good, FAKE, r(v), FAKE, *[r(v)] * 4, FAKE, ws - 1, None) == -3
    for bad in (_view(data=0), _view(data=FAKE + 2), _view(token=60), _view(token=1 << 23)):
        for at in (1, 2):
            args = [v, v, v]
            args[at] = bad
            assert L.mst_block_attention_fwd(s._ref, *[r(x) for x in args], FAKE, r(v), FAKE, FAKE, ws, None) == (-2 if bad.token == 1 << 23 else -1)
            assert L.mst_block_attention_decode(s._ref, *[r(x) for x in args], FAKE, r(v), None, None) == (-2 if bad.token == 1 << 23 else -1)
    assert L.mst_block_attention_fwd(s._ref, *good, FAKE, r(_view(token=0)), FAKE, FAKE, ws, None) == -1     # an output of stride 0
    assert L.mst_block_attention_fwd(None, *good, FAKE, r(v), FAKE, FAKE, ws, None) == -1
    assert L.mst_block_attention_decode(s._ref, None, r(v), r(v), FAKE, r(v), None, None) == -1


def test_empty_calls_do_nothing():
    v = mst.HeadsView(0, 0, 0, 0)
    s, L = _attn(batch=0), mst.lib()
    r = C.byref(v)
    assert L.mst_key_summary(s._ref, r, FAKE, FAKE, 5, None) == 0 and L.mst_block_select(s._ref, r, FAKE, FAKE, FAKE, None) == 0
    assert L.mst_block_attention_decode(s._ref, r, r, r, FAKE, r, None, None) == 0
    assert L.mst_block_attention_fwd(s._ref, r, r, r, FAKE, r, FAKE, FAKE, 1 << 20, None) == 0
    n = _norm(heads=0, kv_heads=0)
    assert L.mst_qk_norm_rotate(C.byref(n), None, None, None, None, FAKE, None, None, None, None) == 0


def test_plans_and_workspaces_stay_in_proportion():
    a, b = (mst.mst_block_plan_bytes(_attn(queries=n, keys=n, batch=2)) for n in (1024, 4096))
    assert 3 * a < b < 5 * a
    # the workspace of a long batch is bounded by what one (batch, key head) needs, or 256 MB and the statistics
    s = _attn(batch=8, queries=16384, keys=16384, heads=16, kv_heads=16, head_dim=128, block=64, n_select=16)
    assert mst.mst_block_attention_workspace_bytes(s, True) < (300 << 20) + 8 * 16 * 16384 * 4
