"""The oracle of the attention half against itself: gradients against differences, summaries against their definition, selection
against a sort, and the planting of a mistake."""
import numpy as np
import pytest

from oracle import attention as oat


@pytest.mark.parametrize("rotated,interleaved", [(8, False), (4, True), (6, False), (0, False)])
def test_gradient_of_norm_and_rotation_is_its_difference(rotated, interleaved):
    rng = np.random.default_rng(1)
    x, dy, w = rng.standard_normal((2, 3, 2, 8)), rng.standard_normal((2, 3, 2, 8)), 1 + 0.1 * rng.standard_normal(8)
    angle = rng.uniform(-3, 3, (2, 3, rotated // 2))
    f = lambda x, w: float((oat.norm_rotate(x, w, np.cos(angle), np.sin(angle), rotated, interleaved, 1e-6) * dy).sum())  # noqa: E731
    dx, dw = oat.norm_rotate_bwd(x, w, np.cos(angle), np.sin(angle), rotated, interleaved, 1e-6, dy)
    h = 1e-6
    for _ in range(10):
        i = tuple(rng.integers(0, n) for n in x.shape)
        e = np.zeros(x.shape)
        e[i] = h
        assert (f(x + e, w) - f(x - e, w)) / (2 * h) == pytest.approx(dx[i], rel=1e-6, abs=1e-7)
    for i in range(8):
        e = np.zeros(8)
        e[i] = h
        assert (f(x, w + e) - f(x, w - e)) / (2 * h) == pytest.approx(dw[i], rel=1e-6, abs=1e-7)


def test_gradients_of_attention_are_its_differences():
    rng = np.random.default_rng(2)
    B, T, H, G, D, block = 1, 70, 4, 2, 8, 32
    q, k, v, d = (rng.standard_normal((B, T, n, D)) for n in (H, G, G, H))
    blocks = np.stack([np.stack([np.array([j for j in (0, t // block) if j <= t // block]) if t >= block else np.array([0, -1]) for t in range(T)])] * G)[None]
    seen = oat.visible(blocks, block, [T], T, T)
    f = lambda q, k, v: float((oat.attention(q, k, v, seen, 0.4)[0] * d).sum())  # noqa: E731
    grads = oat.attention(q, k, v, seen, 0.4, d)[2]
    h = 1e-6
    for n, x in enumerate((q, k, v)):
        for _ in range(4):
            i = tuple(rng.integers(0, s) for s in x.shape)
            e = np.zeros(x.shape)
            e[i] = h
            more, less = [y + e if m == n else y for m, y in enumerate((q, k, v))], [y - e if m == n else y for m, y in enumerate((q, k, v))]
            assert (f(*more) - f(*less)) / (2 * h) == pytest.approx(grads[n][i], rel=1e-5, abs=1e-8)
    # a mistake in the mask is seen: one key more for one row changes that row alone
    wrong = seen.copy()
    wrong[0, 0, 3, 4] = True
    o, other = oat.attention(q, k, v, seen, 0.4)[0], oat.attention(q, k, v, wrong, 0.4)[0]
    assert not np.allclose(o[0, 3, :2], other[0, 3, :2]) and np.array_equal(o[0, 4:], other[0, 4:])


def test_eight_bits():
    s, e = oat.eight_bits(np.array([[1.0, -0.5, 0.0], [1.0, 0.25, 0.0]]))
    assert (s == [64, -8, 0]).all() and e == -6 + 1          # 64 + 64 = 128 -> one shift; (-32 + 16) / 2
    s, e = oat.eight_bits(np.zeros((4, 3)))
    assert (s == 0).all() and e == -106
    s, e = oat.eight_bits(np.array([[np.float64(np.float32(1.9999999)), 1.0]]))
    assert (s == [127, 64]).all() and e == -6                # rounds to 128 and is cut
    s, e = oat.eight_bits(np.array([[0.5 / 64 * 2, 1.5 / 64 * 2, 1.0]]))
    assert (s == [1, 3, 64]).all()
    s, _ = oat.eight_bits(np.array([[2.5 / 64, 3.5 / 64, 1.0]]))
    assert (s == [2, 4, 64]).all()                           # ties to even


def test_selection_of_ties_takes_the_lowest():
    sums, scales = np.ones((1, 1, 6, 8), dtype=np.int8), np.ones((1, 1, 6))
    got = oat.select(np.ones((1, 192, 1, 8)), sums, scales, 32, 3, [192], 1)
    assert got[0, 0, 191].tolist() == [0, 1, 5] and got[0, 0, 0].tolist() == [0, -1, -1] and got[0, 0, 40].tolist() == [0, 1, -1]
    assert oat.counted([3, 2, 5, -1, 9, 7], 7) == [3, 5, 7]
