"""dz of few fp32 tokens, number by number.

With hidden states that are rows of the unit matrix a logit is one number of E, z[t, v] = E[v, t], and dE[v, t] is dz[t, v]: products and sums are exact, and what is left is the error of
exp(z - lse) itself.  Bound, u = 2^-24, y = z - lse with lse as it is given and t = y log2 e: the exponent is rounded once (half a unit of its last place, log 2 of it in the result), log2 e as fp32
holds it is off by 0.22 u of itself, the two exponentials by 2 u each and their products by u each.  Exponentials below 2^-126 are 0."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
from attention_util import DEV  # noqa: E402
from test_gpu_layer_norm import U  # noqa: E402
from test_gpu_vocab_loss import Case  # noqa: E402


@pytest.mark.parametrize("tokens", [1, 8, 33, 64])
def test_probabilities(tokens):
    c = Case(51, tokens, 64, 5000, "f32", labels=np.arange(tokens))
    rng = np.random.default_rng(52)
    c.h.copy_(torch.eye(64, device=DEV)[:tokens])
    c.E.copy_(torch.from_numpy(-rng.uniform(0, 85, (5000, 64))))
    c.E[torch.arange(tokens), torch.arange(tokens)] = 1.0
    c.dloss.fill_(1.0)
    c.forward()
    c.backward(dh=False)
    torch.cuda.synchronize()
    z, lse = c.E.double()[:, :tokens], c.lse.t.double()
    y = z - lse
    t = (y / np.log(2)).abs()
    last = torch.exp2(torch.floor(torch.log2(t.clamp(min=1e-9))) - 23)
    bound = np.log(2) * last / 2 + (0.22 * y.abs() + 6) * U
    bound = bound * torch.exp(y) + 2.0 ** -126
    off = (c.dE.t.double()[:, :tokens] - torch.exp(y)).abs()
    others = torch.ones(5000, tokens, dtype=torch.bool, device=DEV)
    others[torch.arange(tokens), torch.arange(tokens)] = False
    assert (off <= bound)[others].all(), (float((off / bound)[others].max()), int((off > bound)[others].sum()))
    at = torch.expm1(1.0 - lse)
    got = c.dE.t.double()[torch.arange(tokens), torch.arange(tokens)]
    assert ((got - at).abs() <= 4 * U * at.abs() + 2 * U * (1 - lse).abs() * torch.exp(1.0 - lse)).all()
