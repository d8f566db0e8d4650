"""Gradients of the attention over selected blocks, in norms: against differences of the library's own outputs, with a tolerance
that is small beside the gradient, and in bfloat16 against what the kernels' roundings leave, which one rounding more would exceed."""
import numpy as np
import pytest
import torch

from oracle import attention as oat

pytestmark = pytest.mark.gpu
from attention_util import tensor, wide  # noqa: E402
from test_gpu_block_attention import Run, _selection  # noqa: E402


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("D,block,scale", [(32, 32, 0.2), (80, 64, -0.1), (128, 32, 0.09)])
def test_gradients_against_differences(D, block, scale, which):
    rng = np.random.default_rng(D)
    B, T, H, G = 1, 120, 4, 2
    x = {n: tensor(rng.standard_normal((B, T, h, D)), "f32") for n, h in (("q", H), ("k", G), ("v", G))}
    d_o = tensor(rng.standard_normal((B, T, H, D)), "f32")
    blocks = _selection(rng, B, G, T, block, 2, [T])
    run = Run(x["q"], x["k"], x["v"], blocks, block, scale, "f32", None, d_o)
    grad = {"q": run.dq, "k": run.dk, "v": run.dv}[which].double()

    def along(e, h):
        f = []
        for y in (x[which].double() + h * e, x[which].double() - h * e):
            at = dict(x, **{which: y.float()})
            f.append(float((Run(at["q"], at["k"], at["v"], blocks, block, scale, "f32").o.double() * d_o.double()).sum()))
        return (f[0] - f[1]) / (2 * h)
    for i in range(3):
        # the gradient's own direction, where the difference is its length, and two that lie half way to it
        e = grad / grad.norm()
        if i:
            other = torch.from_numpy(rng.standard_normal(e.shape)).to(e)
            e = e + other / other.norm()
        e = e / e.norm()
        h = 2.0 ** -3
        near, far, want = along(e, h), along(e, 2 * h), float((grad * e).sum())
        # a central difference is off by a third of what doubling the step adds (twice that, for the next order), outputs of some
        # roundings each by 2^-22 of their sizes and steps rounded to fp32 by 2^-24 of the inputs, independently of one another
        noise = (2.0 ** -22 * float((run.o.double() * d_o.double()).norm()) + 2.0 ** -24 * float((x[which].double() * grad).norm())) / h
        tolerance = abs(far - near) * 2 / 3 + 4 * noise
        print(D, which, i, want, near, far, tolerance, flush=True)
        assert tolerance < 1e-3 * abs(want)
        assert abs(near - want) <= tolerance


def _rounded(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def _once(x):
    return _rounded(x)


def _twice(x):
    high = _rounded(x)
    return high + _rounded(x - high)


def _modelled(q, k, v, d_o, seen, scale, p_of, ds_of, whole):
    """(o, dq, dk, dv) in 64 bits but for the roundings: p_of and ds_of of P and dS, o and the results to bfloat16; delta from the
    rounded o, `whole`: made up by the sums of dS"""
    B, T, H, D = q.shape
    R = H // k.shape[2]
    out = [np.zeros(x.shape) for x in (q, q, k, v)]
    for h in range(H):
        g = h // R
        s = np.where(seen[0, g], scale * (q[0, :, h] @ k[0, :, g].T), -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o = _rounded(p @ v[0, :, g])
        dp, delta = d_o[0, :, h] @ v[0, :, g].T, (o * d_o[0, :, h]).sum(-1, keepdims=True)
        ds = p * (dp - delta)
        out[0][0, :, h] = o
        out[2][0, :, g] += scale * ds_of(ds).T @ q[0, :, h]
        out[3][0, :, g] += p_of(p).T @ d_o[0, :, h]
        if whole:
            ds = p * (dp - delta - ds.sum(-1, keepdims=True))
        out[1][0, :, h] = scale * ds_of(ds) @ k[0, :, g]
    return [_rounded(x) for x in out]


@pytest.mark.parametrize("D,block", [(64, 32), (64, 64), (128, 64), (40, 128)])
def test_what_the_roundings_of_the_gradients_leave(D, block):
    rng = np.random.default_rng(D + block)
    B, T, H, G, scale = 1, 420, 4, 2, D ** -0.5
    q, d_o, v = (tensor(rng.standard_normal((B, T, n, D)), "bf16") for n in (H, H, G))
    k = tensor(rng.standard_normal((B, T, G, D)) + 2 * rng.standard_normal((1, 1, G, D)), "bf16")       # a direction in common
    blocks = _selection(rng, B, G, T, block, 3, [T])
    run = Run(q, k, v, blocks, block, scale, "bf16", None, d_o)
    seen = oat.visible(blocks, block, [T], T, T)
    arrays = [wide(x) for x in (q, k, v, d_o)]
    exact = oat.attention(*arrays[:3], seen, scale, arrays[3])[2]
    off = lambda got: np.array([np.linalg.norm(a - b) / np.linalg.norm(b) for a, b in zip(got, exact)])  # noqa: E731
    best = off(_modelled(*arrays, seen, scale, _twice, _twice, True)[1:])
    worse = [off(_modelled(*arrays, seen, scale, *kind)[1:]) for kind in ((_once, _once, True), (_twice, _twice, False))]
    # dq would show either lack, dk and dv the roundings
    limit = np.sqrt(best * np.array([min(worse[0][0], worse[1][0]), worse[0][1], worse[0][2]]))
    got = off([wide(x) for x in (run.dq, run.dk, run.dv)])
    print(D, block, "modelled", best, "one rounding", worse[0], "delta of the rounded o", worse[1][0], "limit", limit, "here", got, flush=True)
    assert (limit > 1.05 * best).all()                              # the models can be told apart
    assert (got <= limit).all()
