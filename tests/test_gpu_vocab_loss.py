"""Loss over the vocabulary and its gradients against float64.

Bounds, element by element, before anything is run; u = 2^-24.  A logit is a sum of `width` products (bfloat16: exact ones; fp32: six of each, and what they leave out is below 4.2 u of a term): off by
e_z = (2 width + 8) u sum |h E|.  The log-sum is off by the mean of e_z under p, 200 u for the sums of exponentials and their joints, and 8 u of the sizes of the logits in the exponents; the loss by the
label's own e_z more.  dz is off by |d| p (e_z + e_lse + 8 u (1 + |z| + |lse|)), at the label by |d| p (...) + 2 u |d|, and is rounded to bfloat16 (2^-8 of it in units of the largest dloss; fp32:
three parts, u of it).  Gradients add |dz| times the other factor, and their own sums: a matrix instruction adds 32 products, so n of them
take n / 32 + 32 additions in a row, with six products to a term six times as many; then the output's rounding."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import training_rest as rest

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, space, wide  # noqa: E402
from test_gpu_layer_norm import STEP, U, Out  # noqa: E402


class Case:
    def __init__(self, seed, tokens, width, vocab, dtype, unlabelled=0.2, scale=1.0, labels=None, uniform=False):
        rng = np.random.default_rng(seed)
        self.dtype, self.T, self.W, self.V = dtype, tokens, width, vocab
        self.shape = mst.VocabLossShape(tokens, width, vocab, TYPES[dtype][0])
        kind = TYPES[dtype][1]
        on = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).to(DEV)  # noqa: E731
        self.E = on(rng.standard_normal((vocab, width)) * scale / width ** 0.5, kind)
        self.h = on(rng.standard_normal((tokens, width)), kind)
        lab = rng.integers(0, vocab, tokens)
        lab[rng.random(tokens) < unlabelled] = rng.choice([-100, -1, vocab, vocab + 5])
        self.labels = on(lab if labels is None else labels, torch.int32)
        self.dloss = on(np.full(tokens, 1 / max(tokens, 1)) if uniform else rng.standard_normal(tokens) * 0.1, torch.float32)
        self.loss, self.lse = Out((tokens,), torch.float32), Out((tokens,), torch.float32)
        self.dh, self.dE = Out((tokens, width), kind), Out((vocab, width), kind)
        self.ws = space(mst.mst_vocab_loss_workspace_bytes(self.shape, True) + 64)
        self.ws[-64:] = 99

    def forward(self, stream=None):
        mst.mst_vocab_loss_fwd(self.shape, self.h, self.E, self.labels, self.loss.t, self.lse.t, self.ws[:-64], stream)

    def backward(self, dh=True, dE=True, stream=None):
        mst.mst_vocab_loss_bwd(self.shape, self.h, self.E, self.labels, self.lse.t, self.dloss, self.dh.t if dh else None, self.dE.t if dE else None, self.ws[:-64], stream)

    def check(self, dh=True, dE=True):
        torch.cuda.synchronize()
        for o in (self.loss, self.lse, self.dh, self.dE):
            o.check()
        assert (self.ws[-64:] == 99).all()
        # in float64 on the GPU, where the sizes allow large cases; the formulas are the oracle's
        has = (self.labels >= 0) & (self.labels < self.V)
        h, E, labels, d = self.h[has].double(), self.E.double(), self.labels[has].long(), self.dloss[has].double()
        z = h @ E.T
        lse = torch.logsumexp(z, 1)
        at = torch.arange(len(labels), device=DEV)
        zl = z[at, labels]
        loss = lse - zl
        ez = (2 * self.W + 8) * U * (h.abs() @ E.abs().T)
        p = torch.exp(z - lse[:, None])
        top = z.abs().amax(1) if len(labels) else lse
        elset = (p * ez).sum(1) + 200 * U + 8 * U * (top + zl.abs() + lse.abs())
        for got, ref, bound in ((self.loss, loss, elset + ez[at, labels]), (self.lse, lse, elset)):
            assert (got.t[~has] == 0).all()
            off = (got.t[has].double() - ref).abs()
            assert (off <= bound + U * ref.abs()).all(), float((off - bound).max())
        dz = p * d[:, None]
        edz = dz.abs() * (ez + elset[:, None] + 8 * U * (1 + z.abs() + lse.abs()[:, None]))
        dz[at, labels] -= d
        edz[at, labels] += 4 * U * d.abs()
        edz = edz + (2.0 ** -8 + 2 * U if self.dtype == "bf16" else 4 * U) * dz.abs()
        six = 6 if self.dtype == "f32" else 1
        depth = lambda n: (six * n / 32 + 64) * U + (5 * U if six > 1 else 0)  # noqa: E731
        for wanted, got, a, b, ea, n, rows in ((dh, self.dh, dz, E, edz, self.V, has), (dE, self.dE, dz.T, h, edz.T, len(labels), slice(None))):
            if not wanted:
                continue
            assert got is self.dE or (got.t[~has] == 0).all()
            ref = a @ b
            bound = ea @ b.abs() + depth(n) * (a.abs() @ b.abs())
            bound = bound * (1 + STEP[self.dtype]) + STEP[self.dtype] * ref.abs() + 1e-30
            off = (got.t[rows].double() - ref).abs()
            assert (off <= bound).all(), (got is self.dE, float((off - bound).max()))
        return z


def _all(*a, **kw):
    c = Case(*a, **kw)
    c.forward()
    c.backward()
    c.check()
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 2, 8, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 300, 700])
def test_tokens(tokens, dtype):
    _all(tokens, tokens, 72, 333, dtype, unlabelled=0.2 if tokens > 2 else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 15, 16, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 1000, 5003])
@pytest.mark.parametrize("tokens", [5, 70, 200])
def test_vocabularies(vocab, tokens, dtype):
    _all(vocab, tokens, 64, vocab, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [8, 16, 24, 32, 40, 56, 64, 72, 120, 128, 192, 248, 256, 264, 648, 1280, 2056])
@pytest.mark.parametrize("tokens", [7, 150])
def test_widths(width, tokens, dtype):
    _all(width, tokens, width, 400, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width,vocab", [(2048, 64, 66000), (2100, 128, 30011), (1531, 200, 9001), (4096, 256, 3000 + 11)])
def test_pieces_and_many_tiles(tokens, width, vocab, dtype):
    # (fp32 numbers of 2048 tokens: three pieces of a vocabulary of 66000; bfloat16: two)
    _all(1, tokens, width, vocab, dtype, uniform=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width,vocab", [(1500, 1280, 9003), (1531, 1288, 9001), (600, 264, 30011), (520, 72, 20000), (33, 2056, 9001)])
def test_large_and_small_tiles(tokens, width, vocab, dtype):
    # (all three products by tiles of 256 x 256, by those of 128 x 128 several to a workgroup, and by a mixture)
    _all(17, tokens, width, vocab, dtype, unlabelled=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [9, 100, 400])
def test_labels_far_from_likely(tokens, dtype):
    """logits some hundreds apart: exp(z - z_label) leaves fp32, and so do most probabilities below"""
    c = Case(3, tokens, 64, 700, dtype, scale=60.0)
    c.forward()
    c.backward()
    z = c.check()
    labels = c.labels[(c.labels >= 0) & (c.labels < c.V)].long()
    assert float((z.amax(1) - z[torch.arange(len(labels), device=DEV), labels]).max()) > 150


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [12, 300])
def test_certain_labels(tokens, dtype):
    """losses of 1e-6 and less; the gradient at the label is d (p - 1) without cancellation"""
    c = Case(4, tokens, 64, 500, dtype, unlabelled=0.0)
    c.h.copy_((c.E[c.labels.long()].double() * 25).to(c.h.dtype))
    c.forward()
    c.backward()
    c.check()
    assert float(c.loss.t.median()) < 1e-3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [4, 130, 520])
def test_no_labels(tokens, dtype):
    c = Case(5, tokens, 72, 300, dtype, labels=np.full(tokens, -1))
    c.h.fill_(float("nan"))
    c.dloss.fill_(float("nan"))
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for o in (c.loss, c.lse, c.dh, c.dE):
        o.check()
        assert (o.t == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [20, 150, 600])
def test_what_tokens_without_a_label_hold_counts_for_nothing(tokens, dtype):
    a, b = (Case(6, tokens, 136, 450, dtype, unlabelled=0.5) for _ in range(2))
    out = (b.labels < 0) | (b.labels >= b.V)
    b.h[out] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38] * 34, device=DEV).to(b.h.dtype)
    b.dloss[out] = float("nan")
    for c in (a, b):
        c.forward()
        c.backward()
    torch.cuda.synchronize()
    for x, y in ((a.loss, b.loss), (a.lse, b.lse), (a.dh, b.dh), (a.dE, b.dE)):
        assert torch.equal(x.t, y.t)
    a.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [20, 150, 600])
def test_an_infinite_gradient_is_its_own_token_s_alone(tokens, dtype):
    a, b = (Case(16, tokens, 136, 450, dtype, unlabelled=0.2) for _ in range(2))
    at = [int(t) for t in torch.nonzero((a.labels >= 0) & (a.labels < a.V))[:3, 0]]
    a.dloss[at] = 0.0
    b.dloss[at] = torch.tensor([float("inf"), -float("inf"), float("nan")], device=DEV)
    for c in (a, b):
        c.forward()
        c.backward()
    torch.cuda.synchronize()
    others = torch.ones(tokens, dtype=torch.bool, device=DEV)
    others[at] = False
    assert torch.equal(a.dh.t[others], b.dh.t[others])
    assert not b.dh.t[at].isfinite().any() and b.dE.t.isnan().all()
    a.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_label_for_all(dtype):
    _all(7, 300, 64, 900, dtype, labels=np.full(300, 431))
    _all(8, 40, 64, 900, dtype, labels=np.full(40, 899))


def test_gradients_alone_and_weights_of_zero():
    for dtype in ("f32", "bf16"):
        c = Case(9, 200, 64, 600, dtype)
        c.forward()
        c.dloss[::3] = 0
        c.backward(dE=False)
        torch.cuda.synchronize()
        assert (c.dE.t == 7).all()
        c.backward(dh=False)
        c.check()
        c.dloss.zero_()
        c.backward()
        torch.cuda.synchronize()
        assert (c.dh.t == 0).all() and (c.dE.t == 0).all()


def test_no_tokens():
    for dtype in ("f32", "bf16"):
        shape = mst.VocabLossShape(0, 40, 77, TYPES[dtype][0])
        dE = Out((77, 40), TYPES[dtype][1])
        mst.mst_vocab_loss_fwd(shape, None, None, None, None, None, space(64))
        mst.mst_vocab_loss_bwd(shape, None, None, None, None, None, None, dE.t, space(64))
        torch.cuda.synchronize()
        dE.check()
        assert (dE.t == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_against_the_oracle(dtype):
    c = _all(10, 30, 48, 200, dtype)
    h, E, labels, d = wide(c.h), wide(c.E), c.labels.cpu().numpy(), wide(c.dloss)
    loss, lse = rest.vocab_loss(h, E, labels)
    dh, dE, _ = rest.vocab_loss_bwd(h, E, labels, d)
    off = lambda a, b: float(np.linalg.norm(wide(a.t) - b) / np.linalg.norm(b))  # noqa: E731
    # 2-norms: fp32 sums of tens of terms; bfloat16 outputs and dz are rounded, each by 2^-9 of a norm on average at most
    small = 1e-6 if dtype == "f32" else 2 * 2.0 ** -9
    assert off(c.loss, loss) < 1e-6 and off(c.lse, lse) < 1e-6 and off(c.dh, dh) < small and off(c.dE, dE) < small


@pytest.mark.parametrize("tokens", [40, 300])
def test_gradients_against_differences(tokens):
    """along the gradients themselves, in the kernels' own losses (fp32): a step of 1e-2 of a logit's size leaves 1e-4 of curvature, and losses of 6 hold differences to 2^-20 of the step's"""
    c = Case(11, tokens, 64, 300, "f32", unlabelled=0.1)
    c.dloss.abs_()
    c.forward()
    c.backward()
    d = c.dloss.double()

    def value():
        c.forward()
        torch.cuda.synchronize()
        return float((c.loss.t.double() * d).sum())
    for x, g in ((c.h, c.dh.t.clone()), (c.E, c.dE.t.clone())):
        exact, at = float(g.double().square().sum()), x.clone()
        step = 0.02 / float(g.double().norm())
        x.copy_(at + step * g)
        up = value()
        x.copy_(at - step * g)
        down = value()
        x.copy_(at)
        assert abs((up - down) / (2 * step) - exact) <= 2e-3 * exact


def test_repeated_runs_give_the_same_bits():
    for dtype in ("f32", "bf16"):
        for tokens in (33, 700):
            c = Case(12, tokens, 200, 1500, dtype)
            kept = None
            for _ in range(3):
                c.forward()
                c.backward()
                torch.cuda.synchronize()
                now = [o.t.clone() for o in (c.loss, c.lse, c.dh, c.dE)]
                assert kept is None or all(torch.equal(a, b) for a, b in zip(kept, now))
                kept = now
                c.ws.fill_(255)                                     # nothing is left over from one call for the next: NaN everywhere
                c.ws[-64:] = 99


def test_an_embedding_of_more_than_2_31_numbers():
    W, V = 16384, 140000
    gen = torch.Generator(device=DEV).manual_seed(1)
    E = torch.zeros(V, W, dtype=torch.bfloat16, device=DEV)
    E[-300:] = torch.randn(300, W, generator=gen, device=DEV) * 0.02
    h = torch.randn(3, W, generator=gen, device=DEV).bfloat16()
    labels = torch.tensor([V - 1, V - 300, 5], dtype=torch.int32, device=DEV)
    shape = mst.VocabLossShape(3, W, V, mst.MST_BF16)
    ws = space(mst.mst_vocab_loss_workspace_bytes(shape, True))
    loss, lse, d = (torch.empty(3, device=DEV) for _ in range(3))
    d.fill_(0.5)
    dh, dE = torch.empty_like(h), torch.empty_like(E)
    mst.mst_vocab_loss_fwd(shape, h, E, labels, loss, lse, ws)
    mst.mst_vocab_loss_bwd(shape, h, E, labels, lse, d, dh, dE, ws)
    torch.cuda.synchronize()
    z = h.double() @ E[-300:].double().T                            # the others are 0
    ref = torch.logsumexp(torch.cat([z, torch.full((3, 1), np.log(V - 300.0), dtype=torch.float64, device=DEV)], 1), 1)
    assert ((lse.double() - ref).abs() <= 1e-4 * ref).all()
    p = torch.exp(z - ref[:, None])
    p[0, 299] -= 1
    p[1, 0] -= 1
    off = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert off(dE[-300:], 0.5 * p.T @ h.double()) < 3 * 2.0 ** -9 and off(dh, 0.5 * p @ E[-300:].double()) < 3 * 2.0 ** -9
    rest_p = torch.exp(-ref)
    assert off(dE[7:9], (0.5 * rest_p @ h.double()).expand(2, W)) < 3 * 2.0 ** -9
