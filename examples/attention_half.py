"""The attention half of a GPT-2-like block as a program uses it: sparse products for qkv and proj, norm and rotation of the heads,
attention over selected blocks, the gradients of all of it, and single tokens over a cache.

    python examples/attention_half.py            # a few training steps towards a random target, then eight tokens

The masks of the two products are any sparse masks; their topology updates are the driver's business and are left out here.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2408_11746_amd as mst  # noqa: E402


def angle_table(rows, rotated, device):
    half = rotated // 2
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


class AttentionHalf:
    """y = proj(attention(norm and rotation of qkv(x))) for x [batch, tokens, width], and its gradients."""

    def __init__(self, width, heads, kv_heads, batch, tokens, block=64, n_select=4, density=0.1, device="cuda:0", seed=0):
        self.width, self.heads, self.kv_heads, self.dim = width, heads, kv_heads, width // heads
        self.batch, self.tokens, self.block, self.n_select, self.device = batch, tokens, block, n_select, device
        gen = torch.Generator(device=device).manual_seed(seed)
        rows = (heads + 2 * kv_heads) * self.dim
        self.qkv, self.proj = self._layer(rows, width, density, gen), self._layer(width, width, density, gen)
        self.q_weight, self.k_weight = torch.ones(self.dim, device=device), torch.ones(self.dim, device=device)
        self.table = angle_table(tokens + 64, self.dim, device)
        new = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        B, T, H, G, D, nb = batch, tokens, heads, kv_heads, self.dim, -(-tokens // block)
        self.rows, self.drows = new(B, T, H + 2 * G, D, t=torch.float32), new(B, T, H + 2 * G, D, t=torch.float32)
        self.q, self.k, self.o = new(B, T, H, D), new(B, T, G, D), new(B, T, H, D)
        self.dq, self.dk, self.dv = new(B, T, H, D), new(B, T, G, D), new(B, T, G, D)
        self.y, self.d_o, self.dx = new(B, T, width, t=torch.float32), new(B, T, H, D, t=torch.float32), new(B, T, width, t=torch.float32)
        self.dw_qkv, self.dw_proj = (new(layer.nnz, t=torch.float32) for layer in (self.qkv, self.proj))
        self.dq_weight, self.dk_weight = new(D, t=torch.float32), new(D, t=torch.float32)
        self.sums, self.scales = new(B, G, nb, D, t=torch.int8), new(B, G, nb, t=torch.float32)
        self.blocks, self.lse = new(B, G, T, n_select, t=torch.int32), new(B, H, T, t=torch.float32)
        self.norm = mst.QKNormShape(B, T, H, G, D, D, False, self.table.shape[0], 1e-6, mst.MST_F32, mst.MST_BF16)
        self.shape = mst.BlockAttentionShape(B, T, T, H, G, D, block, n_select, 1 / math.sqrt(D), mst.MST_BF16)
        self.plan = new(mst.mst_block_plan_bytes(self.shape), t=torch.uint8)
        self.ws_attention = new(mst.mst_block_attention_workspace_bytes(self.shape, True), t=torch.uint8)
        self.ws_norm = new(mst.mst_qk_norm_rotate_workspace_bytes(self.norm), t=torch.uint8)

    def _layer(self, O, I, density, gen):
        mask = (torch.rand(O, I, generator=gen, device=self.device) < density).to(torch.uint8)
        weight = torch.randn(O, I, generator=gen, device=self.device) / math.sqrt(density * I)
        count = int(mask.sum())
        layer = mst.Layer(O, I, count, self.device)
        layer.ws = torch.empty(mst.mst_workspace_bytes(O, I, count, self.batch * self.tokens), dtype=torch.uint8, device=self.device)
        layer.load_dense(weight, mask, layer.ws)
        return layer

    def forward(self, x):
        H, G = self.heads, self.kv_heads
        n = self.batch * self.tokens
        mst.mst_sparse_fc_fwd(self.qkv, x, self.rows, n)
        q, k, v = self.rows[:, :, :H], self.rows[:, :, H:H + G], self.rows[:, :, H + G:]
        mst.mst_qk_norm_rotate(self.norm, q, k, self.q_weight, self.k_weight, self.table, None, self.q, self.k)
        self.v = v.to(torch.bfloat16)
        mst.mst_key_summary(self.shape, self.k, self.sums, self.scales, self.tokens)
        mst.mst_block_select(self.shape, self.q, self.sums, self.scales, self.blocks)
        mst.mst_block_plan(self.shape, self.blocks, self.plan)
        mst.mst_block_attention_fwd(self.shape, self.q, self.k, self.v, self.plan, self.o, self.lse, self.ws_attention)
        mst.mst_sparse_fc_fwd(self.proj, self.o, self.y, n, mst.MST_BF16)
        return self.y

    def backward(self, x, dy):
        """dy in bfloat16 (the type of proj's activations); gradients in dx, dw_qkv, dw_proj, dq_weight, dk_weight"""
        H, G = self.heads, self.kv_heads
        n = self.batch * self.tokens
        mst.mst_sparse_fc_bwd(self.proj, dy, self.o, self.d_o, self.dw_proj, n, self.proj.ws, mst.MST_BF16)
        mst.mst_block_attention_bwd(self.shape, self.q, self.k, self.v, self.plan, self.o, self.lse, self.d_o.to(torch.bfloat16),
                                    self.dq, self.dk, self.dv, self.ws_attention)
        q, k = self.rows[:, :, :H], self.rows[:, :, H:H + G]
        mst.mst_qk_norm_rotate_bwd(self.norm, q, k, self.q_weight, self.k_weight, self.table, None, self.dq, self.dk,
                                   self.drows[:, :, :H], self.drows[:, :, H:H + G], self.dq_weight, self.dk_weight, self.ws_norm)
        self.drows[:, :, H + G:] = self.dv
        mst.mst_sparse_fc_bwd(self.qkv, self.drows, x, self.dx, self.dw_qkv, n, self.qkv.ws)
        return self.dx

    def step(self, lr):
        for layer, dw in ((self.qkv, self.dw_qkv), (self.proj, self.dw_proj)):
            layer.values().sub_(lr * dw)
            layer.sync_values()
        self.q_weight.sub_(lr * self.dq_weight)
        self.k_weight.sub_(lr * self.dk_weight)


class Generation:
    """Single tokens after a prompt: a cache of keys, values and summaries that each token extends."""

    def __init__(self, half, capacity):
        if not half.tokens <= capacity <= half.table.shape[0]:          # (positions past the table would take the angles of its last row)
            raise ValueError("a cache of %d tokens: the prompt has %d, the table of angles %d" % (capacity, half.tokens, half.table.shape[0]))
        self.half, self.capacity = half, capacity
        B, H, G, D, dev = half.batch, half.heads, half.kv_heads, half.dim, half.device
        nb = -(-capacity // half.block)
        self.k, self.v = (torch.zeros(B, capacity, G, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.sums, self.scales = torch.zeros(B, G, nb, D, dtype=torch.int8, device=dev), torch.zeros(B, G, nb, device=dev)
        self.k[:, :half.tokens], self.v[:, :half.tokens] = half.k, half.v
        self.lengths = torch.full((B,), half.tokens, dtype=torch.int32, device=dev)
        self.shape = mst.BlockAttentionShape(B, 1, capacity, H, G, D, half.block, half.n_select, 1 / math.sqrt(D), mst.MST_BF16, self.lengths)
        self.norm = mst.QKNormShape(B, 1, H, G, D, D, False, half.table.shape[0], 1e-6, mst.MST_F32, mst.MST_BF16)
        self.q, self.o = (torch.empty(B, 1, H, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.rows = torch.empty(B, 1, H + 2 * G, D, device=dev)
        self.y = torch.empty(B, 1, half.width, device=dev)
        self.blocks = torch.empty(B, G, 1, half.n_select, dtype=torch.int32, device=dev)
        mst.mst_key_summary(self.shape, self.k, self.sums, self.scales, capacity)

    def token(self, x):
        """x [batch, 1, width] -> y; every sequence grows by one"""
        half, at = self.half, int(self.lengths[0])
        if at == self.capacity:
            raise ValueError("the cache is full: %d tokens" % at)
        H, G, B = half.heads, half.kv_heads, half.batch
        mst.mst_sparse_fc_fwd(half.qkv, x, self.rows, B)
        here = slice(at, at + 1)
        mst.mst_qk_norm_rotate(self.norm, self.rows[:, :, :H], self.rows[:, :, H:H + G], half.q_weight, half.k_weight, half.table, self.lengths,
                               self.q, self.k[:, here])
        self.v[:, here] = self.rows[:, :, H + G:]
        self.lengths += 1
        mst.mst_key_summary(self.shape, self.k, self.sums, self.scales, 1)
        mst.mst_block_select(self.shape, self.q, self.sums, self.scales, self.blocks)
        mst.mst_block_attention_decode(self.shape, self.q, self.k, self.v, self.blocks, self.o, None)
        mst.mst_sparse_fc_fwd(half.proj, self.o, self.y, B, mst.MST_BF16)
        return self.y


def main():
    half = AttentionHalf(width=768, heads=12, kv_heads=12, batch=2, tokens=1024)
    gen = torch.Generator(device=half.device).manual_seed(1)
    x, target = (torch.randn(2, 1024, 768, generator=gen, device=half.device) for _ in range(2))
    for i in range(5):
        error = half.forward(x) - target
        print("step %d: mean squared error %.4f" % (i, float(error.square().mean())))
        half.backward(x, (error * (2 / error.numel() * 1e4)).to(torch.bfloat16))
        half.step(2e-3)
    half.forward(x)
    cache = Generation(half, 1024 + 64)
    for i in range(8):
        y = cache.token(torch.randn(2, 1, 768, generator=gen, device=half.device))
    torch.cuda.synchronize()
    print("eight tokens after it; blocks that the last one read: %s" % cache.blocks[0, 0, 0].tolist())


if __name__ == "__main__":
    main()
