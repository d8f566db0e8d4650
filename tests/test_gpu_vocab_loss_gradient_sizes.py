"""Gradients of the loss where dloss differs by most of fp32's range within a batch: one large dloss takes nothing from the gradients of other tokens."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
from attention_util import DEV  # noqa: E402
from test_gpu_vocab_loss import Case  # noqa: E402


@pytest.mark.parametrize("large,small", [(1e30, 1e-15), (3e38, 1e-6), (1e20, 1e-20)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [20, 150, 600])
def test_one_token_far_larger(tokens, dtype, large, small):
    c = Case(41, tokens, 136, 450, dtype, scale=0.1)
    first = int(torch.nonzero((c.labels >= 0) & (c.labels < c.V))[0, 0])
    c.dloss.mul_(small)
    c.dloss[first] = large
    c.forward()
    c.backward(dE=False)
    c.check(dE=False)
    others = torch.arange(tokens, device=DEV) != first
    has = (c.labels >= 0) & (c.labels < c.V) & others
    assert (c.dh.t[has].double().norm(dim=1) > 0).all()


@pytest.mark.parametrize("size", [1e-25, 1e-4, 1.0, 12345.0, 1e30])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_size(dtype, size):
    c = Case(42, 300, 136, 450, dtype, scale=0.1)
    c.dloss.mul_(size)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    # (Case.check adds 1e-30 to its bounds, so that what it looks at is of a size of 1)
    power = float(2.0 ** -np.round(np.log2(size)))
    dh, dE = c.dh.t.double() * power, c.dE.t.double() * power
    one = Case(42, 300, 136, 450, dtype, scale=0.1)
    one.dloss.copy_((c.dloss.double() * power).float())
    assert torch.equal(one.dloss.double(), c.dloss.double() * power)
    one.forward()
    one.backward()
    one.check()
    # the same numbers but for a power of two: everything in between is a product with it, exactly
    assert torch.equal(dh, one.dh.t.double()) and torch.equal(dE, one.dE.t.double())
