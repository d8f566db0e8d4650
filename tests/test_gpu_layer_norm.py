"""Sum of a branch and the residual stream, layer norm of it and its gradients, also from what 8 bits kept, against float64.

Bounds are taken element by element before anything is run.  With u = 2^-24: a row is summed in at most 8 x 4 terms a lane and 6 + 4 levels, so a mean of values is off by 44 u of the mean of their
sizes, the variance (squares, and the same sum) by 48 u of itself, its root and reciprocal by 28 u: n by 44 u r mean|s| + 30 u |n|.  What follows from n is carried along below.  An output is rounded
by half a step of its type, 2^-24 or 2^-8 of its size."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import training_rest as rest

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, space, wide  # noqa: E402

U = 2.0 ** -24
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
GUARD = 64


class Out:
    """An output of n numbers with a guard behind it"""

    def __init__(self, shape, dtype, like=None):
        self.n, self.shape = int(np.prod(shape)), shape
        self.all = torch.full((self.n + GUARD,), 7, dtype=dtype, device=DEV)
        self.t = self.all[:self.n].view(shape)
        if like is not None:
            self.t.copy_(like)

    def check(self):
        assert (self.all[self.n:] == 7).all()


def _given(rng, shape, dtype, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TYPES[dtype][1]).to(DEV)


def _sizes(s, eps):
    """(n, r, bound of n's error) of rows s"""
    _, n, r = rest.layer_norm(s, 1.0, 0.0, eps)
    return n, r, 44 * U * r * np.abs(s).mean(-1, keepdims=True) + 30 * U * np.abs(n) + 2 * U * r * np.abs(s)


def _check_forward(got, s, w, b, eps, y):
    n, r, en = _sizes(s, eps)
    ref = n * w + b
    bound = (np.abs(w) * en + 3 * U * (np.abs(w * n) + np.abs(b))) * (1 + STEP[y]) + STEP[y] * np.abs(ref) + 1e-30
    assert (np.abs(wide(got) - ref) <= bound).all(), float((np.abs(wide(got) - ref) - bound).max())


def _check_backward(got, s, w, eps, dy, ds, x, dw, db):
    n, r, en = _sizes(s, eps)
    dx, rw, rb = rest.layer_norm_bwd(s, w, eps, dy)
    g = dy * w
    mean = lambda a: np.abs(a).mean(-1, keepdims=True)  # noqa: E731
    c1, c2 = g.mean(-1, keepdims=True), (g * n).mean(-1, keepdims=True)
    e2 = 46 * U * mean(g * n) + (np.abs(g) * en).mean(-1, keepdims=True)
    inner = 2 * U * np.abs(g) + 46 * U * mean(g) + np.abs(n) * e2 + en * np.abs(c2) + 4 * U * (np.abs(g) + np.abs(c1) + np.abs(n * c2))
    bound = r * inner + 32 * U * np.abs(dx) + 2 * U * np.abs(ds)
    ref = dx + ds
    bound = bound * (1 + STEP[x]) + STEP[x] * np.abs(ref) + 1e-30
    assert (np.abs(wide(got) - ref) <= bound).all(), float((np.abs(wide(got) - ref) - bound).max())
    # a wavefront's rows one after another, then four wavefronts, 768 / 128 of them and eleven levels
    depth = len(s) / (768 * 4) + 32
    for t, ref, bound in ((dw, rw, depth * U * np.abs(dy * n).sum(0) + (np.abs(dy) * en).sum(0)), (db, rb, depth * U * np.abs(dy).sum(0))):
        if t is not None:
            assert (np.abs(wide(t) - ref) <= bound + 1e-30).all(), float((np.abs(wide(t) - ref) - bound).max())


def _run(seed, rows, width, x="f32", y="f32", dy="f32", kept=False, eps=1e-5, residual=True, weights=True, total="own", ds="own", again=True, sums=True, scale=1.0):
    rng = np.random.default_rng(seed)
    shape = mst.LayerNormShape(rows, width, eps, TYPES[x][0], TYPES[y][0], TYPES[dy][0])
    X = Out((rows, width), TYPES[x][1], _given(rng, (rows, width), x, scale))
    R = Out((rows, width), TYPES[x][1], _given(rng, (rows, width), x, scale)) if residual else None
    w = (1 + 0.3 * rng.standard_normal(width)).astype(np.float32) if weights else np.ones(width, np.float32)
    b = (0.3 * rng.standard_normal(width)).astype(np.float32) if weights else np.zeros(width, np.float32)
    on = lambda a: torch.from_numpy(a).to(DEV) if weights else None  # noqa: E731
    s = X.t.float() + R.t.float() if residual else X.t.float()
    s = s.to(TYPES[x][1])
    S = {"own": lambda: Out((rows, width), TYPES[x][1]), "x": lambda: X, "residual": lambda: R, "none": lambda: None}[total]()
    Y = Out((rows, width), TYPES[y][1])
    codes, units = Out((rows, width), torch.int8), Out((rows, -(-width // 128)), torch.float32)
    keep = mst.Checkpoint8(codes.t, units.t) if kept else None
    W, B = on(w), on(b)
    mst.mst_layer_norm_fwd(shape, X.t, None if R is None else R.t, W, B, None if S is None else S.t, Y.t, keep)
    torch.cuda.synchronize()
    _check_forward(Y.t, wide(s), w.astype(np.float64), b.astype(np.float64), eps, y)
    if S is not None:
        assert torch.equal(S.t, s)
    if kept:
        c, u = rest.keep(s.float().cpu().numpy())
        np.testing.assert_array_equal(codes.t.cpu().numpy(), c)
        np.testing.assert_array_equal(units.t.cpu().numpy(), u)
        s = torch.from_numpy(rest.kept(c, u)).to(DEV)
    DY = _given(rng, (rows, width), dy)
    DS = Out((rows, width), TYPES[x][1], _given(rng, (rows, width), x)) if ds != "none" else None
    given = wide(DS.t) if DS else np.zeros((rows, width))
    DX = DS if ds == "dx" else Out((rows, width), TYPES[x][1])
    DW, DB = (Out((width,), torch.float32), Out((width,), torch.float32)) if sums else (None, None)
    A = Out((rows, width), TYPES[y][1]) if again else None
    get = lambda o: None if o is None else o.t  # noqa: E731
    mst.mst_layer_norm_bwd(shape, None if kept else s, keep, W, B, DY, get(DS), DX.t, get(DW), get(DB), get(A), space(mst.mst_layer_norm_workspace_bytes(shape)))
    torch.cuda.synchronize()
    _check_backward(DX.t, wide(s), w.astype(np.float64), eps, wide(DY), given, x, get(DW), get(DB))
    if again:
        _check_forward(A.t, wide(s), w.astype(np.float64), b.astype(np.float64), eps, y)
    for o in (X, R, S, Y, codes, units, DS, DX, DW, DB, A):
        if o is not None:
            o.check()


WIDTHS = [1, 2, 3, 4, 5, 7, 64, 100, 127, 128, 129, 255, 256, 257, 509, 512, 513, 768, 769, 1001, 1024, 1280, 1283, 1600, 1792, 1793, 2047, 2048, 2049, 2999, 4096, 4097, 5003, 8192, 8193, 12288, 12289,
          16383, 16384]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("kept", [False, True])
def test_widths(width, kept):
    _run(width, 5, width, kept=kept)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("dy", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("width", [130, 767, 2500])
def test_types(x, y, dy, kept, width):
    _run(3, 9, width, x, y, dy, kept)


@pytest.mark.parametrize("rows", [0, 1, 2, 3, 4, 5, 63, 3071, 3073, 7001])
@pytest.mark.parametrize("width", [96, 257])
def test_rows(rows, width):
    _run(rows, rows, width, kept=rows % 2 == 1)


@pytest.mark.parametrize("kw", [dict(residual=False), dict(weights=False), dict(total="x"), dict(total="residual"), dict(total="none"), dict(ds="none"), dict(ds="dx"), dict(again=False), dict(sums=False),
                                dict(residual=False, weights=False, total="none", ds="none", again=False, sums=False), dict(eps=0.0), dict(eps=1.0), dict(scale=1e-12), dict(scale=1e12)], ids=str)
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("width", [300, 2050])
def test_choices(kw, x, width):
    _run(11, 7, width, x, "bf16", "f32", kept=False, **kw)


def test_rows_of_one_value():
    # variance 0: n is 0, and gradients are r (g - mean g)
    shape = mst.LayerNormShape(3, 200, 1e-2, 0, 0, 0)
    s = torch.tensor([[2.0], [0.0], [-65.0]], device=DEV).expand(3, 200).contiguous()
    y, dx = torch.empty_like(s), torch.empty_like(s)
    dy = torch.randn(3, 200, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    mst.mst_layer_norm_fwd(shape, s, None, None, None, None, y)
    mst.mst_layer_norm_bwd(shape, s, None, None, None, dy, None, dx, None, None, None, space(mst.mst_layer_norm_workspace_bytes(shape)))
    torch.cuda.synchronize()
    _check_forward(y, wide(s), 1.0, 0.0, 1e-2, "f32")
    _check_backward(dx, wide(s), 1.0, 1e-2, wide(dy), np.zeros((3, 200)), "f32", None, None)


def test_gradients_of_no_rows_are_zero():
    shape = mst.LayerNormShape(0, 37, 1e-5, 0, 0, 0)
    dw, db = torch.full((37,), 5.0, device=DEV), torch.full((37,), 5.0, device=DEV)
    mst.mst_layer_norm_bwd(shape, None, None, None, None, None, None, None, dw, db, None, space(mst.mst_layer_norm_workspace_bytes(shape)))
    torch.cuda.synchronize()
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("width", [70, 1300])
def test_gradients_against_differences(width):
    """central differences along the gradient itself, in the kernels' own forward: fp32 outputs of size 3 hold the difference of steps of 1e-2 to 1e-5 of it"""
    rng = np.random.default_rng(width)
    rows, shape = 6, mst.LayerNormShape(6, width, 1e-5, 0, 0, 0)
    x = _given(rng, (rows, width), "f32")
    w, b, dy = (torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV) for n in (width, width, (rows, width)))
    dx, dw, db, y = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b), torch.empty_like(x)
    mst.mst_layer_norm_bwd(shape, x, None, w, b, dy, None, dx, dw, db, None, space(mst.mst_layer_norm_workspace_bytes(shape)))

    def value(x, w, b):
        mst.mst_layer_norm_fwd(shape, x, None, w, b, None, y)
        torch.cuda.synchronize()
        return float((y.double() * dy.double()).sum())
    for k, d in enumerate((dx, dw, db)):
        step = 1e-2 / float(d.double().norm())
        at = lambda h: value(*[t + h * d if i == k else t for i, t in enumerate((x, w, b))])  # noqa: E731
        # a central difference of step h along a unit vector is off by h^2 / 6 of third derivatives (below 10 of the gradient here) and by the rounding of the values
        exact = float(d.double().square().sum())
        rounding = 2.0 ** -22 * float((y.double().abs() * dy.double().abs()).sum()) / (width * rows) ** 0.5
        assert abs((at(step) - at(-step)) / (2 * step) - exact) <= 2e-3 * exact + rounding / step, k


def test_more_than_2_31_numbers():
    rows, width = 2_200_000, 1000                                   # bfloat16: offsets of the last rows pass 32 bits
    shape = mst.LayerNormShape(rows, width, 1e-5, 1, 1, 1)
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    last = _given(np.random.default_rng(1), (3, width), "bf16")
    x[-3:] = last
    y, codes, units = torch.empty_like(x), torch.empty(rows, width, dtype=torch.int8, device=DEV), torch.empty(rows, 8, device=DEV)
    kept = mst.Checkpoint8(codes, units)
    mst.mst_layer_norm_fwd(shape, x, None, None, None, None, y, kept)
    torch.cuda.synchronize()
    _check_forward(y[-3:], wide(last), 1.0, 0.0, 1e-5, "bf16")
    c, u = rest.keep(last.float().cpu().numpy())
    np.testing.assert_array_equal(codes[-3:].cpu().numpy(), c)
    np.testing.assert_array_equal(units[-3:].cpu().numpy(), u)
    dx = y                                                          # (taken for both)
    dy = torch.zeros_like(x)
    dy[-3:] = 1 + last
    mst.mst_layer_norm_bwd(shape, None, kept, None, None, dy, None, dx, None, None, None, space(mst.mst_layer_norm_workspace_bytes(shape)))
    torch.cuda.synchronize()
    _check_backward(dx[-3:], rest.kept(c, u).astype(np.float64), 1.0, 1e-5, wide(dy[-3:]), np.zeros((3, width)), "bf16", None, None)
    assert (dx[:5] == 0).all()
