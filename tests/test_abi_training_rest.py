"""Refusals and sizes of norm, activation, 8-bit values and loss that need no GPU: arguments are checked on the host, and these pointers are never read."""
import ctypes as C

import pytest
import torch

import paper_2408_11746_amd as mst

FAKE = 0x10000
KEPT = mst.Checkpoint8(FAKE, FAKE)


class Space:
    """a workspace of so many bytes"""

    def __init__(self, n, at=FAKE):
        self.n, self.at = n, at

    def numel(self):
        return self.n

    def data_ptr(self):
        return self.at


BIG = Space(1 << 40)


def _norm(**kw):
    a = dict(rows=4, width=64, eps=1e-5, in_type=0, out_type=1, grad_type=0)
    a.update(kw)
    return mst.LayerNormShape(*[a[n] for n, _ in mst.LayerNormShape._fields_])


def _gelu(**kw):
    a = dict(rows=4, width=64, erf=0, in_type=0, out_type=1, grad_type=0, in_grad_type=1)
    a.update(kw)
    return mst.GeluShape(*[a[n] for n, _ in mst.GeluShape._fields_])


def _loss(**kw):
    a = dict(tokens=4, width=64, vocab=100, type=1)
    a.update(kw)
    return mst.VocabLossShape(*[a[n] for n, _ in mst.VocabLossShape._fields_])


def _code(call):
    with pytest.raises(mst.MstError) as e:
        call()
    return e.value.code


def _norm_fwd(s, x=FAKE, residual=FAKE, w=FAKE, b=FAKE, total=FAKE, y=FAKE, kept=KEPT):
    mst.mst_layer_norm_fwd(s, x, residual, w, b, total, y, kept, stream=0)


def _norm_bwd(s, total=FAKE, kept=None, w=FAKE, b=FAKE, dy=FAKE, ds=FAKE, dx=FAKE, dw=FAKE, db=FAKE, y=FAKE, ws=BIG):
    mst.mst_layer_norm_bwd(s, total, kept, w, b, dy, ds, dx, dw, db, y, ws, stream=0)


@pytest.mark.parametrize("kw,code", [(dict(rows=-1), -2), (dict(rows=(1 << 31) + 1), -2), (dict(width=0), -2), (dict(width=-5), -2), (dict(width=16385), -2), (dict(eps=-1.0), -1),
                                     (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(in_type=2), -1), (dict(out_type=-1), -1), (dict(grad_type=5), -1)])
def test_norm_refuses_shapes(kw, code):
    s = _norm(**kw)
    assert _code(lambda: _norm_fwd(s)) == code and _code(lambda: _norm_bwd(s)) == code
    assert mst.mst_layer_norm_workspace_bytes(s) == 0


def test_norm_refuses_arguments():
    s = _norm()
    for name in ("x", "y"):
        for bad in (None, FAKE + 4):
            assert _code(lambda: _norm_fwd(s, **{name: bad})) == -1
    for name in ("residual", "w", "b", "total"):
        assert _code(lambda: _norm_fwd(s, **{name: FAKE + 8})) == -1
    for bad in (mst.Checkpoint8(0, FAKE), mst.Checkpoint8(FAKE, 0), mst.Checkpoint8(FAKE + 1, FAKE), mst.Checkpoint8(FAKE, FAKE + 4)):
        assert _code(lambda: _norm_fwd(s, kept=bad)) == -1
        assert _code(lambda: _norm_bwd(s, total=None, kept=bad)) == -1
    for name in ("dy", "dx"):
        for bad in (None, FAKE + 4):
            assert _code(lambda: _norm_bwd(s, **{name: bad})) == -1
    for name in ("total", "w", "b", "ds", "dw", "db", "y"):
        assert _code(lambda: _norm_bwd(s, **{name: FAKE + 8})) == -1
    assert _code(lambda: _norm_bwd(_norm(grad_type=1))) == -1         # in place of dy, of another type
    assert _code(lambda: _norm_bwd(s, total=None)) == -1            # neither the sum nor what was kept of it
    assert _code(lambda: _norm_bwd(s, kept=KEPT)) == -1             # both
    need = mst.mst_layer_norm_workspace_bytes(s)
    assert need > 0
    assert _code(lambda: _norm_bwd(s, ws=Space(need - 1))) == -3
    assert _code(lambda: _norm_bwd(s, ws=Space(need, 0))) == -1
    L = mst.lib()
    assert L.mst_layer_norm_fwd(None, FAKE, None, None, None, None, FAKE, None, None) == -1
    assert L.mst_layer_norm_bwd(None, *[FAKE] * 11, 1 << 30, None) == -1
    _norm_fwd(_norm(rows=0), x=None, y=None, kept=None)             # nothing to do, nothing looked at


@pytest.mark.parametrize("kw,code", [(dict(rows=-1), -2), (dict(width=0), -2), (dict(width=(1 << 24) + 1), -2), (dict(rows=1 << 40, width=1), -2), (dict(rows=(1 << 33) + 1, width=1), -2),
                                     (dict(in_type=2), -1), (dict(out_type=2), -1), (dict(grad_type=2), -1), (dict(in_grad_type=2), -1)])
def test_gelu_refuses_shapes(kw, code):
    s = _gelu(**kw)
    assert _code(lambda: mst.mst_gelu_fwd(s, FAKE, FAKE, None, stream=0)) == code
    assert _code(lambda: mst.mst_gelu_bwd(s, FAKE, None, FAKE, FAKE, None, stream=0)) == code


def test_gelu_refuses_arguments():
    s = _gelu()
    for x, y in ((None, FAKE), (FAKE, None), (FAKE + 4, FAKE), (FAKE, FAKE + 2)):
        assert _code(lambda: mst.mst_gelu_fwd(s, x, y, None, stream=0)) == -1
    assert _code(lambda: mst.mst_gelu_fwd(s, FAKE, FAKE, mst.Checkpoint8(0, FAKE), stream=0)) == -1
    for args in ((None, None, FAKE, FAKE, None), (FAKE, KEPT, FAKE, FAKE, None), (FAKE, None, None, FAKE, None), (FAKE, None, FAKE, None, None), (FAKE + 4, None, FAKE, FAKE + 64, None),
                 (FAKE, None, FAKE, FAKE + 64, FAKE + 8), (None, mst.Checkpoint8(FAKE, 0), FAKE, FAKE + 64, None)):
        assert _code(lambda: mst.mst_gelu_bwd(s, *args, stream=0)) == -1
    assert _code(lambda: mst.mst_gelu_bwd(s, FAKE + 64, None, FAKE, FAKE, None, stream=0)) == -1           # in place, of another type


def test_checkpoint_refuses():
    L, ref = mst.lib(), KEPT._ref
    for rows, width, x, kept, kind, code in ((-1, 8, FAKE, ref, 0, -2), (1, 0, FAKE, ref, 0, -2), (1 << 39, 3, FAKE, ref, 0, -2), (1, 8, None, ref, 0, -1), (1, 8, FAKE + 4, ref, 0, -1),
                                             (1, 8, FAKE, None, 0, -1), (1, 8, FAKE, ref, 3, -1), (1, 8, FAKE, C.byref(mst.Checkpoint8(FAKE, FAKE + 8)._c), 0, -1)):
        assert L.mst_checkpoint_write(rows, width, x, kind, kept, None) == code
        assert L.mst_checkpoint_read(rows, width, kept, kind, x, None) == code
    assert L.mst_checkpoint_write(0, 8, None, 0, ref, None) == 0


def _loss_fwd(s, h=FAKE, E=FAKE, labels=FAKE, loss=FAKE, lse=FAKE, ws=BIG):
    mst.mst_vocab_loss_fwd(s, h, E, labels, loss, lse, ws, stream=0)


def _loss_bwd(s, h=FAKE, E=FAKE, labels=FAKE, lse=FAKE, dloss=FAKE, dh=FAKE, dE=FAKE, ws=BIG):
    mst.mst_vocab_loss_bwd(s, h, E, labels, lse, dloss, dh, dE, ws, stream=0)


@pytest.mark.parametrize("kw,code", [(dict(tokens=-1), -2), (dict(tokens=(1 << 24) + 1), -2), (dict(width=0), -2), (dict(width=12), -2), (dict(width=16392), -2), (dict(vocab=0), -2),
                                     (dict(vocab=(1 << 24) + 1), -2), (dict(type=2), -1)])
def test_loss_refuses_shapes(kw, code):
    s = _loss(**kw)
    assert _code(lambda: _loss_fwd(s)) == code and _code(lambda: _loss_bwd(s)) == code
    assert mst.mst_vocab_loss_workspace_bytes(s, False) == mst.mst_vocab_loss_workspace_bytes(s, True) == 0


def test_loss_refuses_arguments():
    s = _loss()
    for name in ("h", "E", "labels", "lse"):
        for bad in (None, FAKE + 4):
            assert _code(lambda: _loss_fwd(s, **{name: bad})) == -1 and _code(lambda: _loss_bwd(s, **{name: bad})) == -1
    assert _code(lambda: _loss_fwd(s, loss=FAKE + 4)) == -1
    for name in ("dh", "dE"):
        assert _code(lambda: _loss_bwd(s, **{name: FAKE + 4})) == -1
    assert _code(lambda: _loss_bwd(s, dloss=None)) == -1
    for tokens in (4, 300):
        for kind in (0, 1):
            s = _loss(tokens=tokens, type=kind)
            one, both = mst.mst_vocab_loss_workspace_bytes(s, False), mst.mst_vocab_loss_workspace_bytes(s, True)
            assert 0 < one <= both
            assert _code(lambda: _loss_fwd(s, ws=Space(64))) == -3 and _code(lambda: _loss_bwd(s, ws=Space(both // 2))) == -3
    _loss_fwd(_loss(tokens=0), h=None, E=None, labels=None, loss=None, lse=None, ws=Space(0, 0))
    _loss_bwd(_loss(), dh=None, dE=None)                            # nothing is wanted


def test_workspaces_stay_bounded():
    # pieces of the vocabulary of 512 MB, whatever its size; the sums for dh and the packed states beside them
    for kind, size in ((1, 2), (0, 4)):
        for tokens, width, vocab in ((8192, 1280, 50257), (8192, 1280, 1 << 20), (65536, 1024, 50257)):
            n = mst.mst_vocab_loss_workspace_bytes(_loss(tokens=tokens, width=width, vocab=vocab, type=kind), True)
            assert n < (1 << 29) + 64 * tokens * width + 8 * tokens * vocab / 128 + (1 << 24), (kind, tokens, n)
    # the forward of bfloat16 keeps 8 bytes a token and 128 columns
    n = mst.mst_vocab_loss_workspace_bytes(_loss(tokens=8192, width=1280, vocab=50257), False)
    assert n < 8192 * (50257 / 128 + 1) * 8 + 8192 * 1280 * 2 + (1 << 20)


T = torch.zeros(4, 64)


@pytest.mark.parametrize("bad", [torch.zeros(4, 63), torch.zeros(4, 64, dtype=torch.float16), torch.zeros(64, 4).T, torch.zeros(8, 64)[::2], torch.zeros(0)],
                         ids=lambda t: "%s %s" % (t.dtype, tuple(t.shape)))
def test_tensors_have_the_sizes_and_types_of_the_shape(bad):
    s, g, v = _norm(out_type=0), _gelu(out_type=0, in_grad_type=0), _loss(type=0)
    calls = [lambda: _norm_fwd(s, x=bad), lambda: _norm_fwd(s, residual=bad), lambda: _norm_fwd(s, total=bad), lambda: _norm_fwd(s, y=bad), lambda: _norm_fwd(s, w=bad[:, :9] if bad.dim() == 2 else bad),
             lambda: _norm_fwd(s, kept=mst.Checkpoint8(bad, FAKE)), lambda: _norm_bwd(s, total=bad), lambda: _norm_bwd(s, dy=bad), lambda: _norm_bwd(s, ds=bad), lambda: _norm_bwd(s, dx=bad),
             lambda: _norm_bwd(s, y=bad), lambda: mst.mst_gelu_fwd(g, bad, FAKE, None, 0), lambda: mst.mst_gelu_fwd(g, FAKE, bad, None, 0), lambda: mst.mst_gelu_bwd(g, bad, None, FAKE, FAKE, None, 0),
             lambda: mst.mst_gelu_bwd(g, FAKE, None, bad, FAKE, None, 0), lambda: mst.mst_gelu_bwd(g, FAKE, None, FAKE, bad, None, 0), lambda: mst.mst_gelu_bwd(g, FAKE, None, FAKE, FAKE, bad, 0),
             lambda: mst.mst_checkpoint_write(4, 64, bad, 0, KEPT, 0), lambda: mst.mst_checkpoint_read(4, 64, KEPT, 0, bad, 0), lambda: _loss_fwd(v, h=bad), lambda: _loss_fwd(v, E=bad),
             lambda: _loss_fwd(v, labels=bad), lambda: _loss_bwd(v, dh=bad), lambda: _loss_bwd(v, dE=bad), lambda: _loss_bwd(v, h=bad)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_tensors_are_on_the_gpu_that_the_call_runs_on():
    for call in (lambda: _norm_fwd(_norm(), x=T), lambda: mst.mst_gelu_fwd(_gelu(), T, FAKE, None, 0), lambda: _loss_fwd(_loss(type=0), h=T), lambda: mst.mst_checkpoint_write(4, 64, T, 0, KEPT, 0)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_a_checkpoint_is_passed_as_it_is_now():
    kept = mst.Checkpoint8(FAKE, FAKE)
    kept.units = 0                                                  # (once without memory: refused)
    assert _code(lambda: mst.mst_checkpoint_write(1, 8, FAKE, 0, kept, stream=0)) == -1
    kept.codes, kept.units = FAKE + 8, FAKE
    assert _code(lambda: mst.mst_checkpoint_read(1, 8, kept, 0, FAKE, stream=0)) == -1
