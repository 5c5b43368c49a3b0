"""Plain CPU oracle for the AdamW step, with moments as they are or in 8 bits.

TEST INFRASTRUCTURE ONLY (see made_oracle.py for the rules; nothing in the product path imports this).

fp64 numpy, element by element as the step is defined:

    m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2,   g = grad_scale * gradient
    p <- p (1 - lr wd) - lr m c1 / (sqrt(v c2) + eps),   c1 = 1 / (1 - beta1^step),   c2 = 1 / (1 - beta2^step)

8-bit moments: blocks of 256 elements; scale = fp32 of the largest |moment|; m = scale sgn(c) (c / 127)^2, v = scale
(c / 255)^4; the code is the one whose root is nearest (halves up), and at least 1 for a second moment that is not zero.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256


def step(p, g, m, v, lr, beta1, beta2, eps, wd, t, grad_scale=1.0):
    """-> (p, m, v), fp64"""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    c1, c2 = 1.0 / (1.0 - beta1 ** t), 1.0 / (1.0 - beta2 ** t)
    return p * (1.0 - lr * wd) - lr * m * c1 / (np.sqrt(v * c2) + eps), m, v


def unpack(mc, vc, ms, vs):
    """codes [n] and scales [ceil(n / 256)] -> moments, fp64"""
    c, d = np.asarray(mc, np.float64), np.asarray(vc, np.float64)
    at = np.arange(len(c)) // BLOCK
    with np.errstate(invalid="ignore"):
        return np.sign(c) * (c / 127.0) ** 2 * np.asarray(ms, np.float64)[at], (d / 255.0) ** 4 * np.asarray(vs, np.float64)[at]


def pack(m, v):
    """moments [n] -> (codes of m, of v, scales of m, of v)"""
    m, v = np.asarray(m, np.float64), np.asarray(v, np.float64)
    n, blocks = len(m), -(-len(m) // BLOCK)
    mc, vc = np.zeros(n, np.int8), np.zeros(n, np.uint8)
    ms, vs = np.zeros(blocks, np.float32), np.zeros(blocks, np.float32)
    for b in range(blocks):
        r = slice(b * BLOCK, min((b + 1) * BLOCK, n))
        ms[b], vs[b] = np.abs(m[r]).max(), v[r].max()
        if ms[b] > 0:
            c = np.minimum(np.floor(127.0 * np.sqrt(np.abs(m[r]) / np.float64(ms[b])) + 0.5), 127)
            mc[r] = np.sign(m[r]) * c
        if vs[b] > 0:
            c = np.minimum(np.floor(255.0 * (v[r] / np.float64(vs[b])) ** 0.25 + 0.5), 255)
            vc[r] = np.where(v[r] > 0, np.maximum(c, 1), 0)
    return mc, vc, ms, vs
