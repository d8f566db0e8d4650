"""The attention half of a block in float64: norm and rotation of the heads, 8-bit summaries and selection of key blocks,
attention over the selection, and the gradients by their formulas.  Loops and masks, nothing clever.

Arrays are [batch, token, head, head_dim]; a query of n_q sits at position length - n_q + i and sees the keys up to it.
"""
import numpy as np


# ---------------------------------------------------------------- norm and rotation

def _turn(n, angles_cos, angles_sin, rotated, interleaved):
    y = n.copy()
    half = rotated // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = angles_cos[..., i], angles_sin[..., i]
        y[..., a] = n[..., a] * c - n[..., b] * s
        y[..., b] = n[..., a] * s + n[..., b] * c
    return y


def norm_rotate(x, weight, cos, sin, rotated, interleaved, eps):
    """x [B, T, H, D] float64; cos, sin [B, T, rotated / 2] of the tokens' positions."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return _turn(x * r * weight, cos[:, :, None], sin[:, :, None], rotated, interleaved)


def norm_rotate_bwd(x, weight, cos, sin, rotated, interleaved, eps, dy):
    """(dx, dweight)"""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dn = _turn(dy, cos[:, :, None], -sin[:, :, None], rotated, interleaved)
    g = dn * weight
    return r * (g - x * r * r * (g * x).mean(-1, keepdims=True)), (dn * x * r).sum((0, 1, 2))


# ---------------------------------------------------------------- summaries and selection

def eight_bits(members):
    """members [n, D] finite float64 (values of fp32): (8-bit sum over the members, exponent of its unit)."""
    top = np.abs(members).max() if members.size else 0.0
    e = int(np.clip(np.floor(np.log2(top)) if top > 0 else -100, -100, 100))
    if top > 0 and -100 < e < 100:                      # (log2 may be one off next to a power of two)
        e += int(top >= 2.0 ** (e + 1)) - int(top < 2.0 ** e)
    k8 = np.clip(np.rint(members * 2.0 ** (6 - e)), -127, 127)
    s = k8.sum(0)
    peak = int(np.abs(s).max()) if s.size else 0
    shift = max(0, peak.bit_length() - 1 - 6)
    return np.clip(np.rint(s * 2.0 ** -shift), -127, 127).astype(np.int64), e - 6 + shift


def key_summary(k, block, lengths):
    """{(b, g, j): (sums, scale)} of the complete blocks."""
    out = {}
    for b in range(k.shape[0]):
        for g in range(k.shape[2]):
            for j in range(lengths[b] // block):
                s, e = eight_bits(k[b, j * block:(j + 1) * block, g])
                out[b, g, j] = (s, 2.0 ** e)
    return out


def select(q, sums, scales, block, n_select, lengths, kv_heads):
    """blocks [B, G, T, n_select]: own block and the best before it, lowest index on ties, ascending, -1 behind."""
    B, T, H, _ = q.shape
    R = H // kv_heads
    out = np.full((B, kv_heads, T, n_select), -1, dtype=np.int64)
    for b in range(B):
        for g in range(kv_heads):
            for t in range(T):
                p = lengths[b] - T + t
                if p < 0:
                    continue
                own = p // block
                q8, _ = eight_bits(q[b, t, g * R:(g + 1) * R])
                score = [float(q8 @ sums[b, g, j].astype(np.int64)) * float(scales[b, g, j]) for j in range(own)]
                best = sorted(range(own), key=lambda j: (-score[j], j))[:n_select - 1]
                row = sorted(best) + [own]
                out[b, g, t, :len(row)] = row
    return out


def counted(row, own):
    """entries of a selection that count: not negative, up to the own block, above those before them"""
    kept, last = [], -1
    for j in row:
        if last < j <= own:
            kept.append(int(j))
            last = int(j)
    return kept


# ---------------------------------------------------------------- attention

def visible(blocks, block, lengths, n_q, n_k):
    """[B, G, n_q, n_k] booleans"""
    B, G = blocks.shape[:2]
    m = np.zeros((B, G, n_q, n_k), dtype=bool)
    for b in range(B):
        for g in range(G):
            for t in range(n_q):
                p = lengths[b] - n_q + t
                if p < 0:
                    continue
                for j in counted(blocks[b, g, t], p // block):
                    m[b, g, t, j * block:min((j + 1) * block, p + 1)] = True
    return m


def attention(q, k, v, seen, scale, d_o=None):
    """o, lse, and with d_o the gradients (dq, dk, dv) and the sums of absolute values that bound their rounding.  Keys that no
    row sees are not touched."""
    B, T, H, D = q.shape
    G, S = k.shape[2], k.shape[1]
    R = H // G
    o, lse = np.zeros(q.shape), np.full((B, H, T), -np.inf)
    grads = [np.zeros(x.shape) for x in (q, k, v)]
    size = {n: np.zeros(x.shape) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    most = 0.0
    for b in range(B):
        for h in range(H):
            g = h // R
            for t in range(T):
                at = np.nonzero(seen[b, g, t])[0]
                if at.size == 0:
                    continue
                kk, vv = k[b, at, g], v[b, at, g]
                s = scale * (kk @ q[b, t, h])
                most = max(most, abs(scale) * float((np.abs(kk) @ np.abs(q[b, t, h])).max()))
                z = s.max() + np.log(np.exp(s - s.max()).sum())
                p = np.exp(s - z)
                o[b, t, h], lse[b, h, t] = p @ vv, z
                size["o"][b, t, h] = p @ np.abs(vv)
                if d_o is None:
                    continue
                d = d_o[b, t, h]
                dp = vv @ d
                ds = p * (dp - p @ dp)
                spread = p * (np.abs(vv) @ np.abs(d) + p @ (np.abs(vv) @ np.abs(d)))
                grads[0][b, t, h] = scale * ds @ kk
                grads[1][b, at, g] += scale * np.outer(ds, q[b, t, h])
                grads[2][b, at, g] += np.outer(p, d)
                size["dq"][b, t, h] = abs(scale) * spread @ np.abs(kk)
                size["dk"][b, at, g] += abs(scale) * np.outer(spread, np.abs(q[b, t, h]))
                size["dv"][b, at, g] += np.outer(p, np.abs(d))
    return o, lse, grads, size, most
