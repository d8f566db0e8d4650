"""Tensors of heads have the type and at least the sizes that the shape says; nothing here reaches a GPU."""
import pytest
import torch

import paper_2408_11746_amd as mst
from test_abi_attention import FAKE, _attn, _norm

B, T, H, D = 1, 100, 2, 64


def _calls(s, q, k):
    """name -> call with q in place of every tensor of the queries and k of the keys, or of one of them"""
    good = torch.zeros(B, T, H, D, dtype=torch.bfloat16)
    out = []
    for i in range(3):
        out.append(lambda i=i: mst.mst_block_attention_decode(s, q if i == 0 else good, *[k if i == n else good for n in (1, 2)], FAKE, good, None, 0))
    out.append(lambda: mst.mst_block_attention_decode(s, good, good, good, FAKE, q, None, 0))
    out.append(lambda: mst.mst_key_summary(s, k, FAKE, FAKE, 5, 0))
    out.append(lambda: mst.mst_block_select(s, q, FAKE, FAKE, FAKE, 0))
    for i in range(4):
        out.append(lambda i=i: mst.mst_block_attention_fwd(s, *[(q if i in (0, 3) else k) if i == n else good for n in range(3)], FAKE,
                                                           q if i == 3 else good, FAKE, None, 0))
    ws = torch.empty(16, dtype=torch.uint8)
    for i in range(8):                                              # q, k, v, o, d_o, dq, dk, dv
        at = [good] * 8
        at[i] = k if i in (1, 2, 6, 7) else q
        out.append(lambda at=at: mst.mst_block_attention_bwd(s, *at[:3], FAKE, at[3], FAKE, *at[4:], ws, 0))
    return out


BAD = [torch.zeros(B, T, H, D), torch.zeros(B, T, H, D, dtype=torch.float16), torch.zeros(B, T - 1, H, D, dtype=torch.bfloat16),
       torch.zeros(B, T, H - 1, D, dtype=torch.bfloat16), torch.zeros(B, T, H, D - 8, dtype=torch.bfloat16), torch.zeros(0, T, H, D, dtype=torch.bfloat16),
       torch.zeros(T, H, D, dtype=torch.bfloat16), torch.zeros(B, T, H, 2 * D, dtype=torch.bfloat16)[..., ::2]]


@pytest.mark.parametrize("bad", BAD, ids=lambda t: "%s %s" % (t.dtype, tuple(t.shape)))
def test_attention(bad):
    for call in _calls(_attn(), bad, bad):
        with pytest.raises(ValueError):
            call()
    if bad.dim() == 4 and bad.stride(3) == 1:
        view = mst.heads(bad)
        for call in _calls(_attn(), view, view):
            with pytest.raises(ValueError):
                call()


def test_larger_tensors_and_plain_views_pass():
    # refused for another reason: by the library, which looks at alignment
    large = torch.zeros(B + 1, T + 20, H + 1, D + 8, dtype=torch.bfloat16)
    for x in (large, mst.heads(large), mst.HeadsView(large.data_ptr(), 0, 3, 0)):
        with pytest.raises(mst.MstError) as e:
            mst.mst_block_attention_decode(_attn(), x, x, x, FAKE + 1, x, None, 0)
        assert e.value.code == -1


@pytest.mark.parametrize("at", range(8))
def test_norm(at):
    B, T = 1, 4
    f, b = torch.zeros(B, T, H, D), torch.zeros(B, T, H, D, dtype=torch.bfloat16)
    s = _norm(out_type=1)                                           # fp32 to bfloat16
    good = [f, f, b, b, b, b, f, f]                                 # q, k, q_out, k_out; dq_out, dk_out, dq_in, dk_in
    for bad in (b if good[at] is f else f, good[at][:, 1:], good[at][:, :, 1:], good[at][..., 8:], good[at].transpose(2, 3)):
        x = list(good)
        x[at] = bad
        with pytest.raises(ValueError):
            if at < 4:
                mst.mst_qk_norm_rotate(s, x[0], x[1], None, None, FAKE + 1, None, x[2], x[3], 0)
            else:
                mst.mst_qk_norm_rotate_bwd(s, x[0], x[1], None, None, FAKE + 1, None, *x[4:], None, None, torch.empty(1, dtype=torch.uint8), 0)
    # a side without heads is not looked at
    one = _norm(out_type=1, kv_heads=0)
    with pytest.raises(mst.MstError):
        mst.mst_qk_norm_rotate(one, f, b[:, :1], None, None, FAKE + 1, None, b, f[:, :1], 0)


def test_lengths():
    for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            _attn(batch=2, lengths=bad)
    _attn(batch=2, lengths=torch.zeros(2, dtype=torch.int32))
