"""Inputs and bounds of the tests of the attention half.

Bounds are taken element by element from sums of absolute values, before anything is run: a sum of n fp32 products is off by at
most n 2^-24 of the sum of their sizes (here twice that, for the sum's own order and the exponentials), a value rounded
to bfloat16 (8 significant bits, half a unit of the last) by 2^-8 of its size.  A kernel may round to bfloat16 the weights P, (for dK)
dS and each output; the gradients in fact carry P and dS as two numbers and stay well inside.
"""
import numpy as np
import torch

import paper_2408_11746_amd as mst

DEV = "cuda:0"
TYPES = {"f32": (mst.MST_F32, torch.float32), "bf16": (mst.MST_BF16, torch.bfloat16)}


def tensor(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).to(TYPES[dtype][1]).to(DEV)


def wide(t):
    return t.detach().double().cpu().numpy()


def space(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def lengths_of(lengths):
    return torch.tensor(lengths, dtype=torch.int32, device=DEV)


def bounds(ref, size, name, dtype, products, most):
    """largest difference from `ref` that `name` may have; `products`: terms of the longest sum; `most`: largest sum of sizes of a score"""
    fp32 = 2.0 ** -23 * products + 2.0 ** -22 * (most + 8)          # sums, and the scores' error through the exponential
    b = fp32 * size
    if dtype == "bf16":
        if name in ("o", "dv", "dk"):
            b = b + 2.0 ** -8 * size                                # P, or dS
        if name == "dk":
            b = b + 2.0 ** -8 * size                                # delta from the rounded output
        if name == "dq":
            b = b + 2.0 ** -16 * size                               # dS as two numbers
        b = b + 2.0 ** -8 * (np.abs(ref) + b)                       # the output
    return b + 1e-30


def assert_within(got, ref, bound, what):
    over = np.abs(got - ref) - bound
    assert np.isfinite(got).all(), what
    assert (over <= 0).all(), (what, float(over.max()), float(np.abs(got - ref).max()))
