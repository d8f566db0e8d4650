"""What a training step does around products and attention, in float64: layer norm of a sum, the activation, values kept in 8 bits (whose
units and codes are fp32 arithmetic by definition) and the loss over the vocabulary, with the gradients by their formulas."""
import math

import numpy as np

GROUP = 128


# ---------------------------------------------------------------- 8 bits

def keep(x):
    """x [rows, width] fp32 values -> (codes int8, units fp32 [rows, groups])"""
    x = np.asarray(x, dtype=np.float32)
    rows, width = x.shape
    groups = -(-width // GROUP)
    codes, units = np.zeros((rows, width), np.int8), np.zeros((rows, groups), np.float32)
    for g in range(groups):
        v = x[:, g * GROUP:(g + 1) * GROUP]
        unit = np.abs(v).max(1) * np.float32(1 / 127)
        unit = np.maximum(unit, np.float32(2.0 ** -126))
        units[:, g] = unit
        codes[:, g * GROUP:(g + 1) * GROUP] = np.rint(v * (np.float32(1) / unit)[:, None]).astype(np.int8)
    return codes, units


def kept(codes, units):
    """the values in fp32"""
    width = codes.shape[1]
    return codes.astype(np.float32) * np.repeat(units, GROUP, axis=1)[:, :width]


# ---------------------------------------------------------------- layer norm

def layer_norm(s, weight, bias, eps):
    """(y, n, r) of rows s float64"""
    c = s - s.mean(-1, keepdims=True)
    r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    return c * r * weight + bias, c * r, r


def layer_norm_bwd(s, weight, eps, dy):
    """(ds, dweight, dbias)"""
    _, n, r = layer_norm(s, weight, 0.0, eps)
    g = dy * weight
    return r * (g - g.mean(-1, keepdims=True) - n * (g * n).mean(-1, keepdims=True)), (dy * n).sum(0), dy.sum(0)


# ---------------------------------------------------------------- activation

def gelu(x, erf):
    """(value, derivative)"""
    if erf:
        phi = 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-x / math.sqrt(2))
        return x * phi, phi + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-2 * k * (x + 0.044715 * x ** 3)))
    return x * s, s + x * s * (1 - s) * 2 * k * (1 + 3 * 0.044715 * x * x)


# ---------------------------------------------------------------- loss

def has_label(labels, vocab):
    return (labels >= 0) & (labels < vocab)


def vocab_loss(h, E, labels):
    """(loss, lse) [tokens], zeros without a label; rows of h without one are not looked at"""
    loss, lse = np.zeros(len(labels)), np.zeros(len(labels))
    for t in np.flatnonzero(has_label(labels, len(E))):
        z = E @ h[t]
        m = z.max()
        lse[t] = m + math.log(np.exp(z - m).sum())
        loss[t] = lse[t] - z[labels[t]]
    return loss, lse


def vocab_loss_bwd(h, E, labels, dloss):
    """(dh, dE, dz) of sum dloss loss"""
    dz = np.zeros((len(labels), len(E)))
    for t in np.flatnonzero(has_label(labels, len(E))):
        z = E @ h[t]
        p = np.exp(z - z.max())
        dz[t] = dloss[t] * p / p.sum()
        dz[t, labels[t]] -= dloss[t]
    there = has_label(labels, len(E))
    return dz @ E, dz[there].T @ h[there], dz
