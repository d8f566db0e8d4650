"""One training step of a GPT-2-like block with its embedding and its loss, as a program uses the library: layer norms with the residual stream, the attention half, sparse
products around the activation, and the loss over the vocabulary.  What the norms and the activation need again is kept as it is, or in 8 bits.

    python examples/training_step.py            # a few steps on random tokens, with activations kept in 8 bits

The topology updates of the sparse products are left out here (`paper_2408_11746_amd/driver.py` makes them).
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2408_11746_amd as mst  # noqa: E402
from attention_half import AttentionHalf  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


class Norm:
    """Layer norm of stream + branch: the sum (fp32) goes on along the stream, the normed rows (out_type) into a product.  Kept for the backward pass: the sum, or 8 bits of it."""

    def __init__(self, rows, width, out_type, grad_type, keep, device):
        new = lambda *s, t=F32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        types = {F32: mst.MST_F32, BF16: mst.MST_BF16}
        self.shape = mst.LayerNormShape(rows, width, EPS, mst.MST_F32, types[out_type], types[grad_type])
        self.weight, self.bias = torch.ones(width, device=device), torch.zeros(width, device=device)
        self.total, self.y, self.d_total = new(rows, width), new(rows, width, t=out_type), new(rows, width)
        self.d_weight, self.d_bias = new(width), new(width)
        self.kept = mst.Checkpoint8(new(rows, width, t=torch.int8), new(rows, -(-width // 128))) if keep else None
        self.ws = new(mst.mst_layer_norm_workspace_bytes(self.shape), t=torch.uint8)

    def forward(self, stream, branch=None):
        mst.mst_layer_norm_fwd(self.shape, stream, branch, self.weight, self.bias, self.total, self.y, self.kept)
        return self.total, self.y

    def backward(self, dy, d_stream):
        """(with 8 bits also the normed rows again, which the weight gradient of the product behind them reads)"""
        mst.mst_layer_norm_bwd(self.shape, None if self.kept else self.total, self.kept, self.weight, self.bias, dy, d_stream, self.d_total, self.d_weight, self.d_bias,
                               self.y if self.kept else None, self.ws)
        return self.d_total


class Mlp:
    """fc2(gelu(fc1(x))), sparse products of bfloat16 activations"""

    def __init__(self, rows, width, hidden, density, keep, device, seed):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s, t=F32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        self.rows, self.layers = rows, []
        for O, I in ((hidden, width), (width, hidden)):
            mask = (torch.rand(O, I, generator=gen, device=device) < density).to(torch.uint8)
            count = int(mask.sum())
            layer = mst.Layer(O, I, count, device)
            layer.ws = new(mst.mst_workspace_bytes(O, I, count, rows), t=torch.uint8)
            layer.load_dense(torch.randn(O, I, generator=gen, device=device) / math.sqrt(density * I), mask, layer.ws)
            layer.dw = new(count)
            self.layers.append(layer)
        self.shape = mst.GeluShape(rows, hidden, 0, mst.MST_F32, mst.MST_BF16, mst.MST_F32, mst.MST_BF16)
        self.pre, self.act, self.d_act, self.d_pre = new(rows, hidden), new(rows, hidden, t=BF16), new(rows, hidden), new(rows, hidden, t=BF16)
        self.out, self.dx = new(rows, width), new(rows, width)
        self.kept = mst.Checkpoint8(new(rows, hidden, t=torch.int8), new(rows, -(-hidden // 128))) if keep else None

    def forward(self, x):
        fc1, fc2 = self.layers
        mst.mst_sparse_fc_fwd(fc1, x, self.pre, self.rows, mst.MST_BF16)
        mst.mst_gelu_fwd(self.shape, self.pre, self.act, self.kept)
        mst.mst_sparse_fc_fwd(fc2, self.act, self.out, self.rows, mst.MST_BF16)
        return self.out

    def backward(self, d_out):
        """gradient of x; fc1's weight gradient is fc1_weight's, once x is there again"""
        fc1, fc2 = self.layers
        d_out = d_out.to(BF16)
        mst.mst_sparse_fc_bwd_input(fc2, d_out, self.d_act, self.rows, mst.MST_BF16)
        if self.kept:
            mst.mst_gelu_bwd(self.shape, None, self.kept, self.d_act, self.d_pre, self.act)      # (the activation again: it need not have been kept)
        else:
            mst.mst_gelu_bwd(self.shape, self.pre, None, self.d_act, self.d_pre)
        mst.mst_sparse_fc_bwd_weight(fc2, d_out, self.act, fc2.dw, self.rows, fc2.ws, mst.MST_BF16)
        mst.mst_sparse_fc_bwd_input(fc1, self.d_pre, self.dx, self.rows, mst.MST_BF16)
        return self.dx

    def fc1_weight(self, x):
        fc1 = self.layers[0]
        mst.mst_sparse_fc_bwd_weight(fc1, self.d_pre, x, fc1.dw, self.rows, fc1.ws, mst.MST_BF16)


class Model:
    """embedding -> norm -> attention half -> norm -> mlp -> norm -> loss"""

    def __init__(self, vocab, width, heads, batch, tokens, keep=True, density=0.3, block=64, device="cuda:0", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.rows, self.width, self.vocab = batch * tokens, width, vocab
        self.embedding = torch.randn(vocab, width, generator=gen, device=device)
        self.output = (torch.randn(vocab, width, generator=gen, device=device) / math.sqrt(width)).to(BF16)
        self.attention = AttentionHalf(width, heads, heads, batch, tokens, block=block, n_select=3, density=density, device=device, seed=seed + 1)
        self.mlp = Mlp(self.rows, width, 4 * width, density, keep, device, seed + 2)
        self.norms = [Norm(self.rows, width, out, grad, keep, device) for out, grad in ((F32, F32), (BF16, F32), (BF16, BF16))]
        self.shape = mst.VocabLossShape(self.rows, width, vocab, mst.MST_BF16)
        new = lambda *s, t=F32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
        self.loss, self.lse = new(self.rows), new(self.rows)
        self.dh, self.d_output = new(self.rows, width, t=BF16), new(vocab, width, t=BF16)
        self.ws = new(mst.mst_vocab_loss_workspace_bytes(self.shape, True), t=torch.uint8)

    def forward(self, ids, labels):
        """ids, labels int32 [rows]; a label outside the vocabulary is none.  Losses of the tokens, 0 without a label."""
        first, second, last = self.norms
        stream, y = first.forward(self.embedding[ids.long()])
        a = self.attention.forward(y.view(self.attention.batch, self.attention.tokens, self.width))
        stream, y = second.forward(stream, a)
        stream, h = last.forward(stream, self.mlp.forward(y))
        mst.mst_vocab_loss_fwd(self.shape, h, self.output, labels, self.loss, self.lse, self.ws)
        return self.loss

    def backward(self, ids, labels, d_loss):
        first, second, last = self.norms
        # (the last norm's rows are read by the loss before its backward pass may write them again)
        mst.mst_vocab_loss_bwd(self.shape, last.y, self.output, labels, self.lse, d_loss, self.dh, self.d_output, self.ws)
        d = last.backward(self.dh, None)
        dx = self.mlp.backward(d)
        d = second.backward(dx, d)
        self.mlp.fc1_weight(second.y)
        half = self.attention
        dx = half.backward(first.y.view(half.batch, half.tokens, self.width), d.view(half.batch, half.tokens, self.width).to(BF16))
        d = first.backward(dx, d)
        self.d_embedding = torch.zeros_like(self.embedding).index_add_(0, ids.long(), d)

    def step(self, lr):
        self.attention.step(lr)
        for layer in self.mlp.layers:
            layer.values().sub_(lr * layer.dw)
            layer.sync_values()
        for norm in self.norms:
            norm.weight.sub_(lr * norm.d_weight)
            norm.bias.sub_(lr * norm.d_bias)
        self.embedding.sub_(lr * self.d_embedding)
        self.output.copy_(self.output.float() - lr * self.d_output)


def main():
    model = Model(vocab=5000, width=512, heads=8, batch=2, tokens=512)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    ids = torch.randint(0, 5000, (model.rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    labels = torch.roll(ids, -1)
    labels[511::512] = -100                                         # (the last token of a sequence predicts nothing)
    count = int((labels >= 0).sum())
    for i in range(6):
        loss = model.forward(ids, labels)
        print("step %d: loss %.4f" % (i, float(loss.sum()) / count))
        model.backward(ids, labels, torch.full((model.rows,), 1 / count, device="cuda:0"))
        model.step(0.5)


if __name__ == "__main__":
    main()
