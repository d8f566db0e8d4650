"""The example program: forward and gradients of the attention half with its sparse products, and single tokens after a prompt that
agree with the prompt's own rows."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from attention_half import AttentionHalf, Generation  # noqa: E402


def _dense(layer):
    W = torch.empty(layer.O, layer.I, device="cuda:0")
    layer.export_dense(W)
    return W.double()


def _reference(half, x, dy):
    """torch's differentiation in 64 bits, over the selection that the program made"""
    B, T, H, G, D = half.batch, half.tokens, half.heads, half.kv_heads, half.dim
    x = x.double().requires_grad_()
    w = [_dense(half.qkv).requires_grad_(), _dense(half.proj).requires_grad_()]
    rows = (x @ w[0].T).view(B, T, H + 2 * G, D)
    half_d = D // 2
    cos, sin = half.table[:T, None, :half_d].double(), half.table[:T, None, half_d:].double()

    def turned(t):
        n = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)
        a, b = n[..., :half_d], n[..., half_d:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    q, k, v = turned(rows[:, :, :H]), turned(rows[:, :, H:H + G]), rows[:, :, H + G:]
    nb = half.sums.shape[2]
    chosen = torch.zeros(B, G, T, nb + 1, dtype=torch.bool, device=x.device)
    chosen.scatter_(3, torch.where(half.blocks < 0, nb, half.blocks).long(), True)
    seen = chosen[..., :nb].repeat_interleave(half.block, 3)[..., :T] & torch.ones(T, T, dtype=torch.bool, device=x.device).tril()
    r = H // G
    s = torch.einsum("bthd,bshd->bhts", q, k.repeat_interleave(r, 2)) / D ** 0.5
    p = torch.softmax(s.masked_fill(~seen.repeat_interleave(r, 1), -1e300), -1)
    y = torch.einsum("bhts,bshd->bthd", p, v.repeat_interleave(r, 2)).reshape(B, T, -1) @ w[1].T
    return [y] + list(torch.autograd.grad(y, (x, *w), dy.double()))


@pytest.mark.parametrize("heads,kv_heads,tokens,block", [(4, 4, 200, 32), (6, 2, 150, 64)])
def test_training_step(heads, kv_heads, tokens, block):
    half = AttentionHalf(width=heads * 64, heads=heads, kv_heads=kv_heads, batch=2, tokens=tokens, block=block, n_select=3, density=0.3, seed=3)
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    x = torch.randn(2, tokens, half.width, generator=gen, device="cuda:0")
    dy = torch.randn(2, tokens, half.width, generator=gen, device="cuda:0").to(torch.bfloat16)
    y = half.forward(x)
    dx = half.backward(x, dy)
    torch.cuda.synchronize()
    ref = _reference(half, x, dy)
    masks = []
    for layer in (half.qkv, half.proj):
        M = torch.empty(layer.O, layer.I, dtype=torch.uint8, device="cuda:0")
        layer.export_dense(None, M)
        masks.append(M.bool())
    got = [y, dx, half.dw_qkv, half.dw_proj]
    want = [ref[0], ref[1], ref[2][masks[0]], ref[3][masks[1]]]
    # 2-norms: a handful of bfloat16 roundings (2^-9 of a norm each on average) in a row, half of them met twice on the way back
    for name, a, b, roundings in zip(("y", "dx", "dw_qkv", "dw_proj"), got, want, (4, 10, 10, 5)):
        off = float((a.double() - b).norm() / b.norm())
        print(name, off, flush=True)
        assert off <= roundings * 2.0 ** -9 + 2e-4, (name, off)


def test_tokens_after_a_prompt_agree_with_the_prompt():
    B, T, more = 2, 96, 40                                          # a block ends among the tokens
    full = AttentionHalf(width=256, heads=4, kv_heads=2, batch=B, tokens=T + more, block=32, n_select=3, density=0.3, seed=5)
    part = AttentionHalf(width=256, heads=4, kv_heads=2, batch=B, tokens=T, block=32, n_select=3, density=0.3, seed=5)
    x = torch.randn(B, T + more, 256, generator=torch.Generator(device="cuda:0").manual_seed(6), device="cuda:0")
    y = full.forward(x)
    part.forward(x[:, :T].contiguous())
    cache = Generation(part, T + more)
    for i in range(more):
        got = cache.token(x[:, T + i:T + i + 1].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(cache.blocks[:, :, 0], full.blocks[:, :, T + i]), i
        off = float((got[:, 0] - y[:, T + i]).norm() / y[:, T + i].norm())
        assert off <= 4 * 2.0 ** -9, (i, off)                       # weights in fp32 here, in bfloat16 there; one more rounding of o
    np.testing.assert_array_equal(cache.lengths.cpu().numpy(), T + more)
