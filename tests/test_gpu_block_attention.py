"""Attention over selected blocks, forward, backward and for single tokens, against float64."""
import numpy as np
import pytest
import torch

import paper_2408_11746_amd as mst
from oracle import attention as oat

pytestmark = pytest.mark.gpu
from attention_util import DEV, TYPES, assert_within, bounds, lengths_of, space, tensor, wide  # noqa: E402


def _selection(rng, B, G, T, block, n_select, lengths, wild=False):
    """random ascending selections; `wild`: entries that do not count among them, and rows that leave the own block out"""
    out = np.full((B, G, T, n_select), -1, dtype=np.int32)
    for b in range(B):
        for g in range(G):
            for t in range(T):
                p = lengths[b] - T + t
                if p < 0 and not wild:
                    continue
                own = max(p, 0) // block
                if wild:
                    out[b, g, t] = rng.integers(-3, own + 4, n_select)
                else:
                    row = sorted(set(rng.permutation(own)[:n_select - 1].tolist()) | {own})
                    out[b, g, t, :len(row)] = row
    return out


class Run:
    def __init__(self, q, k, v, blocks, block, scale, dtype, lengths=None, d_o=None, decode=False):
        B, T, H, D = q.shape
        S, G = k.shape[1], k.shape[2]
        self.shape = mst.BlockAttentionShape(B, T, S, H, G, D, block, blocks.shape[3], scale, TYPES[dtype][0], None if lengths is None else lengths_of(lengths))
        self.o, self.lse = torch.full_like(q, float("nan")), torch.full((B, H, T), float("nan"), device=DEV)
        blocks = torch.from_numpy(np.ascontiguousarray(blocks)).to(DEV)
        if decode:
            mst.mst_block_attention_decode(self.shape, q, k, v, blocks, self.o, self.lse)
        else:
            self.plan, self.ws = space(mst.mst_block_plan_bytes(self.shape)), space(mst.mst_block_attention_workspace_bytes(self.shape, d_o is not None))
            mst.mst_block_plan(self.shape, blocks, self.plan)
            mst.mst_block_attention_fwd(self.shape, q, k, v, self.plan, self.o, self.lse, self.ws)
        if d_o is not None:
            self.dq, self.dk, self.dv = (torch.full_like(x, float("nan")) for x in (q, k, v))
            mst.mst_block_attention_bwd(self.shape, q, k, v, self.plan, self.o, self.lse, d_o, self.dq, self.dk, self.dv, self.ws)
        torch.cuda.synchronize()


def _check(run, q, k, v, blocks, block, scale, dtype, lengths, d_o=None):
    B, T, H, D = q.shape
    S = k.shape[1]
    seen = oat.visible(blocks, block, lengths, T, S)
    kept = [np.where(np.arange(S)[None, :, None, None] < np.asarray(lengths)[:, None, None, None], wide(x), 0) for x in (k, v)]
    o, lse, grads, size, most = oat.attention(wide(q), kept[0], kept[1], seen, scale, None if d_o is None else wide(d_o))
    n = D + int(seen.sum(-1).max(initial=0))
    assert_within(wide(run.o), o, bounds(o, size["o"], "o", dtype, n, most), "o")
    got = wide(run.lse)
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got), empty)
    assert (np.abs(got[~empty] - lse[~empty]) <= 2.0 ** -22 * (most + n + np.abs(lse[~empty]) + 4)).all()
    if d_o is None:
        return
    rows = int(seen.sum(2).max(initial=0)) * (H // k.shape[2])
    for name, g, got in zip(("dq", "dk", "dv"), grads, (run.dq, run.dk, run.dv)):
        terms = n + D if name == "dq" else rows + 2 * D + n
        assert_within(wide(got), g, bounds(g, size[name], name, dtype, terms, most), name)


SHAPES = [
    # B, T, S, H, G, D, block, n_select, lengths
    (1, 1, 1, 1, 1, 64, 64, 1, None),
    (1, 64, 64, 2, 2, 64, 64, 1, None),
    (2, 130, 130, 2, 1, 64, 32, 3, None),
    (2, 150, 150, 6, 2, 40, 32, 3, [150, 77]),                      # three heads to a key head, left-padded
    (1, 200, 200, 3, 3, 128, 64, 2, None),
    (1, 300, 300, 4, 1, 96, 128, 2, None),
    (2, 33, 290, 8, 2, 80, 64, 3, [290, 131]),                      # a piece of a prompt over a longer cache
    (1, 129, 129, 20, 1, 16, 32, 4, None),                          # twenty heads: rows that straddle wavefronts
    (1, 70, 70, 64, 1, 8, 32, 2, None),
    (3, 40, 70, 1, 1, 24, 32, 2, [70, 0, 5]),                       # no keys at all; fewer than queries
    (1, 260, 260, 1, 1, 128, 128, 3, None),
    (1, 500, 500, 2, 2, 32, 64, 8, None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,S,H,G,D,block,n_select,lengths", SHAPES)
def test_forward_and_gradients(B, T, S, H, G, D, block, n_select, lengths, dtype):
    rng = np.random.default_rng(T * S + D)
    n = lengths or [S] * B
    # keys with a direction in common, as heads have: what falls out of dQ
    common = rng.standard_normal((1, 1, G, D))
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, T, H, D)), dtype)
    k, v = tensor(rng.standard_normal((B, S, G, D)) + common, dtype), tensor(rng.standard_normal((B, S, G, D)), dtype)
    blocks = _selection(rng, B, G, T, block, n_select, n)
    scale = D ** -0.5
    run = Run(q, k, v, blocks, block, scale, dtype, lengths, d_o)
    _check(run, q, k, v, blocks, block, scale, dtype, n, d_o)
    few = Run(q, k, v, blocks, block, scale, dtype, lengths, decode=True)
    # (the single-token form keeps its weights in fp32: within the same bound)
    _check(few, q, k, v, blocks, block, scale, dtype, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selections_of_any_kind(dtype):
    rng = np.random.default_rng(5)
    B, T, S, H, G, D, block, n_select = 2, 160, 160, 4, 2, 64, 32, 5
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, T, H, D)), dtype)
    k, v = tensor(rng.standard_normal((B, S, G, D)), dtype), tensor(rng.standard_normal((B, S, G, D)), dtype)
    lengths = [160, 100]
    blocks = _selection(rng, B, G, T, block, n_select, lengths, wild=True)
    blocks[0, 0, 3] = -1                                            # an empty row
    blocks[0, 1, :, 0] = 0                                          # a block that every query reads
    blocks[1, 0, 50] = [2 ** 31 - 1, -2 ** 31, 0, 0, 1]
    run = Run(q, k, v, blocks, block, 0.3, dtype, lengths, d_o)
    _check(run, q, k, v, blocks, block, 0.3, dtype, lengths, d_o)
    few = Run(q, k, v, blocks, block, 0.3, dtype, lengths, decode=True)
    _check(few, q, k, v, blocks, block, 0.3, dtype, lengths)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_is_read_past_a_sequence(dtype):
    rng = np.random.default_rng(6)
    B, T, S, H, G, D, block, n_select = 2, 60, 200, 2, 1, 64, 64, 2
    lengths = [100, 129]
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), dtype), tensor(rng.standard_normal((B, T, H, D)), dtype)
    k, v = tensor(rng.standard_normal((B, S, G, D)), dtype), tensor(rng.standard_normal((B, S, G, D)), dtype)
    blocks = _selection(rng, B, G, T, block, n_select, lengths)
    clean = Run(q, k, v, blocks, block, 0.125, dtype, lengths, d_o)
    for b, n in enumerate(lengths):
        k[b, n:], v[b, n:] = float("nan"), float("inf")
    run = Run(q, k, v, blocks, block, 0.125, dtype, lengths, d_o)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(run, name), getattr(clean, name)), name
    for b, n in enumerate(lengths):
        assert (run.dk[b, n:] == 0).all() and (run.dv[b, n:] == 0).all()
    assert torch.equal(Run(q, k, v, blocks, block, 0.125, dtype, lengths, decode=True).o, Run(q, k.nan_to_num(), v.nan_to_num(posinf=0), blocks, block, 0.125, dtype, lengths, decode=True).o)


@pytest.mark.parametrize("scale", [-0.7, 0.0, 30.0])
def test_scales(scale):
    rng = np.random.default_rng(8)
    B, T, H, G, D, block = 1, 100, 2, 1, 32, 32
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), "f32"), tensor(rng.standard_normal((B, T, H, D)), "f32")
    k, v = tensor(rng.standard_normal((B, T, G, D)), "f32"), tensor(rng.standard_normal((B, T, G, D)), "f32")
    blocks = _selection(rng, B, G, T, block, 2, [T])
    run = Run(q, k, v, blocks, block, scale, "f32", None, d_o)
    _check(run, q, k, v, blocks, block, scale, "f32", [T], d_o)
    _check(Run(q, k, v, blocks, block, scale, "f32", decode=True), q, k, v, blocks, block, scale, "f32", [T])


def test_scores_that_rise_block_after_block():
    # the running maximum is left behind and taken up again; late weights would overflow against an early one
    rng = np.random.default_rng(9)
    B, T, D, block = 1, 256, 64, 32
    k = np.repeat(np.arange(T // block), block)[None, :, None, None] * np.ones((1, 1, 1, D)) * 3.0
    q, v = np.ones((B, T, 1, D)), rng.standard_normal((B, T, 1, D))
    blocks = _selection(rng, B, 1, T, block, 8, [T])
    for sign in (1.0, -1.0):
        for dtype in ("f32", "bf16"):
            qt, kt, vt = tensor(sign * q, dtype), tensor(k, dtype), tensor(v, dtype)
            run = Run(qt, kt, vt, blocks, block, 1.0, dtype)
            _check(run, qt, kt, vt, blocks, block, 1.0, dtype, [T])


def test_layouts():
    rng = np.random.default_rng(10)
    B, T, H, G, D, block = 2, 90, 4, 2, 64, 32
    base = [tensor(rng.standard_normal((B, T, n, D)), "bf16") for n in (H, G, G, H)]
    blocks = _selection(rng, B, G, T, block, 2, [T] * B)
    plain = Run(*base[:3], blocks, block, 0.125, "bf16", None, base[3])
    heads_first = [x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in base]
    rows = torch.zeros(B, T + 3, H + 2 * G + 1, D, dtype=torch.bfloat16, device=DEV)
    for x, at in zip(base[:3], (0, H, H + G)):
        rows[:, 3:, at:at + x.shape[2]] = x
    fused = [rows[:, 3:, :H], rows[:, 3:, H:H + G], rows[:, 3:, H + G:H + 2 * G], base[3].transpose(0, 1).contiguous().transpose(0, 1)]
    for other in (heads_first, fused):
        run = Run(*other[:3], blocks, block, 0.125, "bf16", None, other[3])
        for name in ("o", "lse", "dq", "dk", "dv"):
            assert torch.equal(getattr(run, name), getattr(plain, name)), name
    # one key head for all sequences, by a stride of 0
    shared = [base[1][:1].expand(B, T, G, D), base[2][:1].expand(B, T, G, D)]
    run, copy = Run(base[0], *shared, blocks, block, 0.125, "bf16"), Run(base[0], *[x.contiguous() for x in shared], blocks, block, 0.125, "bf16")
    assert torch.equal(run.o, copy.o)


def test_offsets_past_32_bits():
    # a cache of 2.3e9 elements of which few are read: the last sequences lie past 2^31 elements and 2^32 bytes
    B, S, G, D, block, n_select = 9, 131072, 16, 128, 128, 3
    assert B * S * G * D > 2 ** 31
    k, v = (torch.zeros(B, S, G, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rng = np.random.default_rng(12)
    lengths = [S] * B
    blocks = np.tile(np.array([5, 700, 1023], dtype=np.int32), (B, G, 1, 1))
    at = np.concatenate([np.arange(j * block, (j + 1) * block) for j in blocks[0, 0, 0]])
    small = [tensor(rng.standard_normal((B, at.size, G, D)), "bf16") for _ in range(2)]
    k[:, torch.from_numpy(at).to(DEV)], v[:, torch.from_numpy(at).to(DEV)] = small
    q = tensor(rng.standard_normal((B, 1, G, D)), "bf16")
    near = np.tile(np.array([0, 1, 2], dtype=np.int32), (B, G, 1, 1))
    want = Run(q, *small, near, block, 0.1, "bf16", decode=True)
    got = Run(q, k, v, blocks, block, 0.1, "bf16", lengths, decode=True)
    assert torch.equal(got.o, want.o) and torch.equal(got.lse, want.lse)
    got, want = Run(q, k, v, blocks, block, 0.1, "bf16", lengths), Run(q, *small, near, block, 0.1, "bf16")
    assert torch.equal(got.o, want.o) and torch.equal(got.lse, want.lse)


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(13)
    B, T, H, G, D, block, n_select = 2, 700, 4, 2, 64, 32, 6
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), "bf16"), tensor(rng.standard_normal((B, T, H, D)), "bf16")
    k, v = tensor(rng.standard_normal((B, T, G, D)), "bf16"), tensor(rng.standard_normal((B, T, G, D)), "bf16")
    shape = mst.BlockAttentionShape(B, T, T, H, G, D, block, n_select, 0.125, mst.MST_BF16)
    nb = -(-T // block)

    def buffers():
        return dict(sums=torch.zeros(B, G, nb, D, dtype=torch.int8, device=DEV), scales=torch.zeros(B, G, nb, device=DEV),
                    blocks=torch.zeros(B, G, T, n_select, dtype=torch.int32, device=DEV), o=torch.empty_like(q), lse=torch.empty(B, H, T, device=DEV),
                    dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v), plan=space(mst.mst_block_plan_bytes(shape)),
                    ws=space(mst.mst_block_attention_workspace_bytes(shape, True)))

    def step(x, stream=None):
        mst.mst_key_summary(shape, k, x["sums"], x["scales"], T, stream)
        mst.mst_block_select(shape, q, x["sums"], x["scales"], x["blocks"], stream)
        mst.mst_block_plan(shape, x["blocks"], x["plan"], stream)
        mst.mst_block_attention_fwd(shape, q, k, v, x["plan"], x["o"], x["lse"], x["ws"], stream)
        mst.mst_block_attention_bwd(shape, q, k, v, x["plan"], x["o"], x["lse"], d_o, x["dq"], x["dk"], x["dv"], x["ws"], stream)
    a, b, c = buffers(), buffers(), buffers()
    step(a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    step(b, s)
    s.synchronize()
    names = ("sums", "scales", "blocks", "o", "lse", "dq", "dk", "dv")
    assert all(torch.equal(a[n], b[n]) for n in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c)
    for _ in range(3):
        for n in names:
            c[n].zero_()
        step(b)                                                     # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], c[n]) for n in names)


def test_gradients_against_differences():
    # through the library itself, in fp32: central differences of <o, d> along random directions
    rng = np.random.default_rng(14)
    B, T, H, G, D, block = 1, 120, 4, 2, 32, 32
    q, d_o = tensor(rng.standard_normal((B, T, H, D)), "f32"), tensor(rng.standard_normal((B, T, H, D)), "f32")
    k, v = tensor(rng.standard_normal((B, T, G, D)), "f32"), tensor(rng.standard_normal((B, T, G, D)), "f32")
    blocks = _selection(rng, B, G, T, block, 2, [T])
    run = Run(q, k, v, blocks, block, 0.2, "f32", None, d_o)
    h = 2.0 ** -7
    for n, grad in enumerate((run.dq, run.dk, run.dv)):
        x = [q, k, v]
        e = torch.randn_like(x[n])
        e /= e.norm()
        up = Run(*[y + h * e if m == n else y for m, y in enumerate(x)], blocks, block, 0.2, "f32").o
        down = Run(*[y - h * e if m == n else y for m, y in enumerate(x)], blocks, block, 0.2, "f32").o
        diff = float(((up.double() - down.double()) * d_o.double()).sum()) / (2 * h)
        want = float((grad.double() * e.double()).sum())
        # the third derivative of <o, d> along a unit direction is below ~10 |d| here: h^2/6 of it, and fp32 outputs over 2h
        assert abs(diff - want) <= h * h / 6 * 10 * float(d_o.norm()) + 2.0 ** -22 * float(d_o.norm()) * float(run.o.norm()) / h


def test_few_queries_of_no_sequence():
    q, k = torch.zeros(0, 1, 2, 64, device=DEV), torch.zeros(0, 8, 2, 64, device=DEV)
    run = Run(q, k, k, np.zeros((0, 2, 1, 1), dtype=np.int32), 32, 1.0, "f32", decode=True)
    assert run.o.numel() == 0
    # a cache without keys: every row is empty, forward, single-token and gradient
    q, k = torch.randn(2, 3, 2, 64, device=DEV), torch.zeros(2, 0, 2, 64, device=DEV)
    run = Run(q, k, k, np.zeros((2, 2, 3, 1), dtype=np.int32), 32, 1.0, "f32", None, q)
    assert (run.o == 0).all() and torch.isneginf(run.lse).all() and (run.dq == 0).all()
    assert (Run(q, k, k, np.zeros((2, 2, 3, 1), dtype=np.int32), 32, 1.0, "f32", decode=True).o == 0).all()


def test_gradients_of_many_key_heads_over_a_long_cache():
    # more than the workspace takes at a time: the key heads go in two groups, to the same bits as heads by themselves
    T, S, G, D, block, n_select = 64, 262144, 24, 8, 128, 4
    torch.manual_seed(16)
    q, d_o = (torch.randn(1, T, G, D, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(1, S, G, D, device=DEV).bfloat16() for _ in range(2))
    rng = np.random.default_rng(16)
    nb = S // block
    before = np.sort(rng.integers(0, nb - 1, (1, G, T, n_select - 1)), axis=-1)     # some twice
    blocks = np.concatenate([before, np.full((1, G, T, 1), nb - 1)], axis=-1).astype(np.int32)
    shape = mst.BlockAttentionShape(1, T, S, G, G, D, block, n_select, 0.3, mst.MST_BF16)
    one = mst.BlockAttentionShape(1, T, S, 1, 1, D, block, n_select, 0.3, mst.MST_BF16)
    assert mst.mst_block_attention_workspace_bytes(shape, True) < 20 * mst.mst_block_attention_workspace_bytes(one, True)      # (not 24)
    run = Run(q, k, v, blocks, block, 0.3, "bf16", None, d_o)
    for g in (0, 14, 15, 23):
        head = [x[:, :, g:g + 1].contiguous() for x in (q, k, v, d_o)]
        alone = Run(*head[:3], blocks[:, g:g + 1], block, 0.3, "bf16", None, head[3])
        for name in ("o", "dq", "dk", "dv"):
            assert torch.equal(getattr(run, name)[:, :, g:g + 1], getattr(alone, name)), (g, name)
