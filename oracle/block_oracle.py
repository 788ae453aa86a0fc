"""CPU oracle of the layer in a transformer block: the norms around it, its form for a few tokens and the hidden
activations kept in 8 bits.  The paper has none of these: the definitions are this library's (include/locmoe.h).

TEST INFRASTRUCTURE ONLY: only the tests may import this file; the product path never does, and this file imports nothing
from it.  NumPy float64, one function per definition; the gradients are pinned in tests/test_block_oracle_pins.py by
central differences of the forward functions, the forward functions by sums written out.
"""
from __future__ import annotations

import numpy as np

from oracle import locmoe_backward_oracle as bwd
from oracle import locmoe_oracle as fwd


def _ones(gamma, d):
    return np.ones(d) if gamma is None else np.asarray(gamma, dtype=np.float64)


def norm(v, eps):
    """v r and r = 1 / sqrt(mean v^2 + eps), row by row."""
    v = np.asarray(v, dtype=np.float64)
    r = 1.0 / np.sqrt(np.mean(v * v, axis=1) + eps)
    return v * r[:, None], r


def norm_gate(x, gamma, eps, E):
    """xn = x r gamma, r, and the mean of every block of d/E features of xn."""
    n, r = norm(x, eps)
    xn = n * _ones(gamma, n.shape[1])
    return xn, r, xn.reshape(len(xn), E, -1).mean(axis=2)


def combine_norm(out, slot, w, res, gamma, post_norm, eps, scale):
    """y = res + scale w gamma n(out[slot]) (n: the norm, or nothing), y = res where slot < 0; and r (0 there)."""
    y = np.array(res, dtype=np.float64)
    r = np.zeros(len(slot))
    g = _ones(gamma, y.shape[1])
    for m in np.nonzero(np.asarray(slot) >= 0)[0]:
        o = np.asarray(out[slot[m]], dtype=np.float64)
        r[m] = 1.0 / np.sqrt(np.mean(o * o) + eps) if post_norm else 1.0
        y[m] += scale * w[m] * g * o * r[m]
    return y, r


def norm_backward(dn, v, r):
    """Gradient with respect to v of a loss whose gradient with respect to v r is dn (r depends on v)."""
    n = v * r[:, None]
    return r[:, None] * (dn - n * np.mean(dn * n, axis=1, keepdims=True))


def combine_norm_backward(dy, out, slot, w, gamma, post_norm, scale, r):
    """dout (zeros where no token's row is), dw, dgamma."""
    dy, out = np.asarray(dy, dtype=np.float64), np.asarray(out, dtype=np.float64)
    d = dy.shape[1]
    g = _ones(gamma, d)
    dout, dw, dgamma = np.zeros_like(out), np.zeros(len(slot)), np.zeros(d)
    kept = np.nonzero(np.asarray(slot) >= 0)[0]
    rows = np.asarray(slot)[kept]
    o, wk, rk = out[rows], np.asarray(w, dtype=np.float64)[kept], np.asarray(r, dtype=np.float64)[kept]
    n = o * rk[:, None] if post_norm else o
    branch = scale * dy[kept]
    dw[kept] = np.sum(branch * g * n, axis=1)
    dgamma[:] = np.sum(branch * wk[:, None] * n, axis=0)
    dn = branch * g * wk[:, None]
    dout[rows] = norm_backward(dn, o, rk) if post_norm else dn
    return dout, dw, dgamma


def dispatch_norm_backward(dsend, slot, dg, x, gamma, r, dres):
    """dx and dgamma of the norm ahead of the layer, for dxn = dsend[slot] (kept) + (E/d) dg."""
    x, r = np.asarray(x, dtype=np.float64), np.asarray(r, dtype=np.float64)
    dxn = bwd.dispatch_backward(np.asarray(dsend, dtype=np.float64), np.asarray(slot)) + bwd.gate_backward(dg, x.shape[1])
    dx = norm_backward(dxn * _ones(gamma, x.shape[1]), x, r)
    if dres is not None:
        dx = dx + np.asarray(dres, dtype=np.float64)
    return dx, np.sum(dxn * x * r[:, None], axis=0)


def layer_few(x, g32, eps, relu, C, weights):
    """The layer, a token at a time: eid, w, slot (m or -1) and the experts' outputs (zeros for dropped tokens)."""
    eid, w, _, _ = fwd.route(g32, eps, relu)
    out = np.zeros((len(x), np.shape(x)[1]))
    slot = np.full(len(x), -1)
    for m in range(len(x)):
        if int(np.sum(eid[:m] == eid[m])) < C:
            slot[m] = m
            out[m] = fwd.ffn_rows(np.asarray(x[m:m + 1]), *weights(int(eid[m])))[0]
    return eid, w, slot, out


def bf16(v):
    """Rounded to bf16, to nearest, ties to even (finite values)."""
    b = np.ascontiguousarray(v, dtype=np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


def to8(z):
    """(q, unit): blocks of 16 columns of a row as whole numbers of at most 127 and a bf16 unit."""
    z = np.asarray(z, dtype=np.float64)
    blocks = np.pad(z, ((0, 0), (0, -z.shape[1] % 16))).reshape(len(z), -1, 16)
    unit = bf16(np.max(np.abs(blocks), axis=2) / 127.0)
    q = np.rint(blocks / np.where(unit > 0, unit, 1.0)[:, :, None])
    return q.reshape(len(z), -1)[:, :z.shape[1]], unit


def from8(q, unit):
    return np.asarray(q, dtype=np.float64) * np.repeat(unit, 16, axis=1)[:, :np.shape(q)[1]]
