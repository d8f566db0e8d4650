"""The activation between fc1 and fc2 and its gradient, values in 8 bits, and the one from the other, against float64.

Bounds, element by element, u = 2^-24.  The exponent t = 2 log2(e) u(x) is off by 6 u |t| (the cube, its factor, the sum, two products), the exponential by 0.7 of that and one unit of its last
place, 2 u, the reciprocal by 2 u and the sum under it by u: the logistic s by s ((1 - s)(5 u |t| + 2 u) + 3 u).  Its share in the derivative is carried along.  erfc is given 16 u of itself."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import training_rest as rest

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, wide  # noqa: E402
from test_gpu_layer_norm import STEP, U, Out  # noqa: E402

TINY = 1e-35                                                        # exponentials below 2^-126 are 0


def _bounds(x, erf):
    """largest errors of value and derivative before they are rounded"""
    y, slope = rest.gelu(x, erf)
    c = np.clip(x, -30, 30)
    if erf:
        density = np.exp(-c * c / 2) * 0.3989422804
        ephi = 2 * U * np.abs(c) * density + 16 * U * np.abs(y / np.where(x == 0, 1, x)) + U
        term = np.abs(c) * density
        return np.abs(x) * ephi + U * np.abs(y) + TINY, ephi + term * (4 * U * 0.72 * c * c + 6 * U) + U * np.abs(slope) + TINY
    k = 0.7978845608
    t = np.abs(2 * 1.442695 * k * (c + 0.044715 * c ** 3))
    s = 1 / (1 + np.exp(-2 * k * (c + 0.044715 * c ** 3)))
    es = s * ((1 - s) * (5 * U * t + 2 * U) + 3 * U)
    factor = np.abs(c) * 2 * k * (1 + 3 * 0.044715 * c * c)
    return np.abs(x) * es + U * np.abs(y) + TINY, es + factor * (es * (1 - s) + s * (es + U)) + 6 * U * factor * s * (1 - s) + U * np.abs(slope) + TINY


def _within(got, ref, bound, kind):
    bound = bound * (1 + STEP[kind]) + STEP[kind] * np.abs(ref)
    assert (np.abs(wide(got) - ref) <= bound).all(), float((np.abs(wide(got) - ref) - bound).max())


def _run(seed, rows, width, erf, x="f32", y="f32", dy="f32", dx="f32", kept=False, again=True, in_place=False, values=None):
    rng = np.random.default_rng(seed)
    shape = mst.GeluShape(rows, width, erf, *[TYPES[t][0] for t in (x, y, dy, dx)])
    v = rng.standard_normal((rows, width)) * 3 if values is None else values
    X = torch.from_numpy(v).to(TYPES[x][1]).to(DEV)
    Y, codes, units = Out((rows, width), TYPES[y][1]), Out((rows, width), torch.int8), Out((rows, -(-width // 128)), torch.float32)
    keep = mst.Checkpoint8(codes.t, units.t) if kept else None
    mst.mst_gelu_fwd(shape, X, Y.t, keep)
    torch.cuda.synchronize()
    at = wide(X)
    _within(Y.t, rest.gelu(at, erf)[0], _bounds(at, erf)[0], y)
    if kept:
        c, u = rest.keep(X.float().cpu().numpy())
        np.testing.assert_array_equal(codes.t.cpu().numpy(), c)
        np.testing.assert_array_equal(units.t.cpu().numpy(), u)
        at = rest.kept(c, u).astype(np.float64)
    D = Out((rows, width), TYPES[dy][1], torch.from_numpy(rng.standard_normal((rows, width))).to(DEV))
    given = wide(D.t)
    G = D if in_place else Out((rows, width), TYPES[dx][1])
    A = Out((rows, width), TYPES[y][1]) if again else None
    mst.mst_gelu_bwd(shape, None if kept else X, keep, D.t, G.t, A.t if again else None)
    torch.cuda.synchronize()
    eb = _bounds(at, erf)
    _within(G.t, given * rest.gelu(at, erf)[1], np.abs(given) * eb[1] + U * np.abs(given), dx)
    if again:
        _within(A.t, rest.gelu(at, erf)[0], eb[0], y)
    for o in (Y, codes, units, D, G, A):
        if o is not None:
            o.check()


@pytest.mark.parametrize("erf", [False, True])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows,width", [(0, 5), (1, 1), (1, 3), (3, 1), (7, 5), (1, 128), (2, 127), (3, 129), (5, 384), (33, 2047), (4, 5120), (1000, 130)])
def test_sizes(rows, width, erf, kept):
    _run(rows + width, rows, width, erf, kept=kept)


@pytest.mark.parametrize("types", [(a, b, c, d) for a in ("f32", "bf16") for b in ("f32", "bf16") for c in ("f32", "bf16") for d in ("f32", "bf16")])
@pytest.mark.parametrize("erf", [False, True])
@pytest.mark.parametrize("kept", [False, True])
def test_types(types, erf, kept):
    _run(5, 6, 261, erf, *types, kept=kept)


@pytest.mark.parametrize("erf", [False, True])
def test_everywhere(erf):
    v = np.concatenate([np.linspace(-12, 12, 2001), [0.0, -0.0, 1e-30, -1e-30, 2.0 ** -126, 100, -100, 29.9, -29.9, 30.1, -30.1, 1e10, -1e10, 3e38, -3e38]])
    _run(6, 1, len(v), erf, values=v[None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_without_the_value(dtype):
    _run(7, 5, 700, False, dy=dtype, dx=dtype, in_place=True, again=False)
    _run(8, 5, 700, False, dy=dtype, dx=dtype, in_place=True, kept=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(0, 3), (1, 1), (2, 127), (3, 128), (3, 129), (70, 1601), (4096, 768)])
def test_write_and_read(rows, width, dtype):
    rng = np.random.default_rng(rows + width)
    x = torch.from_numpy(rng.standard_normal((rows, width)) * 10.0 ** rng.uniform(-20, 20, (rows, 1))).to(TYPES[dtype][1]).to(DEV)
    codes, units, back = Out((rows, width), torch.int8), Out((rows, -(-width // 128)), torch.float32), Out((rows, width), TYPES[dtype][1])
    kept = mst.Checkpoint8(codes.t, units.t)
    mst.mst_checkpoint_write(rows, width, x, TYPES[dtype][0], kept)
    mst.mst_checkpoint_read(rows, width, kept, TYPES[dtype][0], back.t)
    torch.cuda.synchronize()
    c, u = rest.keep(x.float().cpu().numpy())
    np.testing.assert_array_equal(codes.t.cpu().numpy(), c)
    np.testing.assert_array_equal(units.t.cpu().numpy(), u)
    assert torch.equal(back.t, torch.from_numpy(rest.kept(c, u)).to(TYPES[dtype][1]).to(DEV))
    for o in (codes, units, back):
        o.check()


def test_extremes_in_8_bits():
    x = torch.zeros(8, 130, device=DEV)
    x[0, 5] = 3e38
    x[1] = 1e-45                                                    # the smallest number there is
    x[2, :3] = torch.tensor([1e-37, -1e-38, 5e-40])
    x[3, 128] = -2.5                                                # alone in a group of two
    x[4, 0] = float("inf")
    x[5, 127] = float("-inf")
    x[6, 40] = float("nan")
    codes, units, back = torch.empty(8, 130, dtype=torch.int8, device=DEV), torch.empty(8, 2, device=DEV), torch.empty(8, 130, device=DEV)
    kept = mst.Checkpoint8(codes, units)
    mst.mst_checkpoint_write(8, 130, x, mst.MST_F32, kept)
    mst.mst_checkpoint_read(8, 130, kept, mst.MST_F32, back)
    torch.cuda.synchronize()
    fine = [0, 1, 2, 3, 7]
    c, u = rest.keep(x[fine].cpu().numpy())
    np.testing.assert_array_equal(codes[fine].cpu().numpy(), c)
    np.testing.assert_array_equal(units[fine].cpu().numpy(), u)
    for r in (4, 5, 6):                                             # what is not finite shows in its whole group, and in no other
        assert back[r, :128].isnan().all() and (back[r, 128:] == 0).all()


def test_more_than_2_31_numbers():
    rows, width = 1_100_000, 2001                                   # offsets and groups behind 2^31
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    last = torch.randn(2, width, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    x[-2:] = last
    shape = mst.GeluShape(rows, width, 0, 1, 1, 1, 1)
    y, codes, units = torch.empty_like(x), torch.empty(rows, width, dtype=torch.int8, device=DEV), torch.empty(rows, 16, device=DEV)
    kept = mst.Checkpoint8(codes, units)
    mst.mst_gelu_fwd(shape, x, y, kept)
    mst.mst_gelu_bwd(shape, None, kept, x, x, None)                  # in place
    torch.cuda.synchronize()
    _within(y[-2:], rest.gelu(wide(last), 0)[0], _bounds(wide(last), 0)[0], "bf16")
    c, u = rest.keep(last.float().cpu().numpy())
    np.testing.assert_array_equal(codes[-2:].cpu().numpy(), c)
    at = rest.kept(c, u).astype(np.float64)
    _within(x[-2:], wide(last) * rest.gelu(at, 0)[1], np.abs(wide(last)) * (_bounds(at, 0)[1] + U), "bf16")
    assert (x[:3] == 0).all()


def test_more_than_2_34_numbers():
    rows, width = 2 ** 22 + 5, 4096                                 # more groups than a launch has half wavefronts
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    x[-3:] = torch.randn(3, width, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    codes, units = torch.empty(rows, width, dtype=torch.int8, device=DEV), torch.empty(rows, 32, device=DEV)
    kept = mst.Checkpoint8(codes, units)
    mst.mst_checkpoint_write(rows, width, x, mst.MST_BF16, kept)
    torch.cuda.synchronize()
    c, u = rest.keep(x[-3:].float().cpu().numpy())
    np.testing.assert_array_equal(codes[-3:].cpu().numpy(), c)
    np.testing.assert_array_equal(units[-3:].cpu().numpy(), u)
    assert not codes[:-3].any()
    last = x[-3:].clone()
    mst.mst_checkpoint_read(rows, width, kept, mst.MST_BF16, x)
    torch.cuda.synchronize()
    assert torch.equal(x[-3:], torch.from_numpy(rest.kept(c, u)).bfloat16().to(DEV))
    x[-3:] = last
    mst.mst_gelu_bwd(mst.GeluShape(rows, width, 0, 1, 1, 1, 1), None, kept, x, x, None)
    torch.cuda.synchronize()
    at = rest.kept(c, u).astype(np.float64)
    _within(x[-3:], wide(last) * rest.gelu(at, 0)[1], np.abs(wide(last)) * (_bounds(at, 0)[1] + U), "bf16")
    y = codes = units = kept = None
    y = torch.empty_like(x)
    x[-3:] = last
    mst.mst_gelu_fwd(mst.GeluShape(rows, width, 0, 1, 1, 1, 1), x, y)
    torch.cuda.synchronize()
    _within(y[-3:], rest.gelu(wide(last), 0)[0], _bounds(wide(last), 0)[0], "bf16")
