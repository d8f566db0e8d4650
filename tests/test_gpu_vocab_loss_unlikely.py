"""Losses of tokens whose label is some 84 to 100 nats less likely than all others together, by tiles: sums of exponentials relative to the label's logit leave fp32 there, some of them only
when the sums of all columns meet.  Against float64, with the bounds of test_gpu_vocab_loss.py."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
from attention_util import DEV  # noqa: E402
from test_gpu_vocab_loss import Case  # noqa: E402

V = 50257
# What the label's logit is below the others', from and to, and the log-sum of those.  (The small random logits have a deviation of 0.1, so that a loss is within 1 of the sum of both.)
MASSES = {"even": (73.0, 90.0, 10.82), "two parts": (83.5, 100.0, 1.0), "one above": (73.0, 90.0, 100.0)}


class Unlikely(Case):
    """Column 0 of h is 1, so that column 0 of E is a logit of its own beside small random ones.  (Numbers that bfloat16 holds, but for one.)"""

    def __init__(self, tokens, dtype, mass):
        rng = np.random.default_rng(20)
        labels = 6000 + rng.permutation(V - 6000)[:tokens]
        labels[rng.random(tokens) < 0.1] = -1
        super().__init__(21, tokens, 64, V, dtype, scale=0.1, labels=labels)
        self.at = self.labels[self.labels >= 0].long()
        self.h[:, 0] = 1
        self.E[:, 0] = -128 if mass == "two parts" else 0
        if mass == "two parts":
            self.E[5:7, 0] = 0
            self.E[5000, 0] = -0.35
        if mass == "one above":
            self.E[777, 0] = 100


@pytest.mark.parametrize("mass", MASSES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [70, 1500])
def test_unlikely_labels(tokens, dtype, mass):
    # (70 tokens: tiles of 128 x 128, 1500 of 256 x 256.  All labels of a call are equally far: a row whose sum leaves fp32 has its neighbours' formed again too.)
    c = Unlikely(tokens, dtype, mass)
    first, last, log_sum = MASSES[mass]
    for below in np.arange(first, last + 0.5, 0.5):
        c.E[c.at, 0] = -float(below)
        c.forward()
        c.backward()
        losses = c.loss.t[c.labels >= 0]
        assert ((losses - (below + log_sum)).abs() < 1).all(), (below, float(losses.min()), float(losses.max()))
        c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [70, 1500])
def test_labels_unlikely_by_different_amounts(tokens, dtype):
    c = Unlikely(tokens, dtype, "even")
    c.E[c.at, 0] = -(60 + 0.5 * (torch.arange(len(c.at), device=DEV) % 80)).to(c.E.dtype)
    c.forward()
    c.backward()
    c.check()
