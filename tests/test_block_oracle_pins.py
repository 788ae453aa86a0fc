"""The block oracle against what does not depend on it: sums written out, central differences, PyTorch's reverse mode."""
import math

import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from oracle import locmoe_oracle as orc


def test_norm_gate_by_hand():
    x = np.array([[3.0, 4.0, 0.0, 0.0], [1.0, -1.0, 1.0, -1.0]])
    xn, r, g = blk.norm_gate(x, np.array([1.0, 2.0, 3.0, 4.0]), 0.0, 2)
    assert np.allclose(r, [0.4, 1.0])            # mean squares 25/4 and 1
    assert np.allclose(xn, [[1.2, 3.2, 0.0, 0.0], [1.0, -2.0, 3.0, -4.0]])
    assert np.allclose(g, [[2.2, 0.0], [-0.5, -0.5]])


def test_combine_norm_by_hand():
    out = np.array([[3.0, 4.0], [6.0, 8.0]])
    res = np.array([[10.0, 20.0], [30.0, 40.0]])
    y, r = blk.combine_norm(out, np.array([1, -1]), np.array([0.5, 0.9]), res, None, True, 0.0, 2.0)
    r0 = 1.0 / math.sqrt(50.0)
    assert np.allclose(r, [r0, 0.0]) and np.allclose(y, [[10.0 + 6.0 * r0, 20.0 + 8.0 * r0], [30.0, 40.0]])
    y, r = blk.combine_norm(out, np.array([1, -1]), np.array([0.5, 0.9]), res, np.array([1.0, 10.0]), False, 0.0, 2.0)
    assert np.allclose(y[0], [16.0, 100.0]) and r[0] == 1.0


def problem(seed, T=5, d=12, E=3, rows=6):
    rng = np.random.default_rng(seed)
    slot = np.array([4, -1, 0, 2, -1])
    return rng, dict(x=rng.standard_normal((T, d)), out=rng.standard_normal((rows, d)), w=rng.uniform(0.1, 1, T),
                     gi=rng.uniform(0.5, 1.5, d), go=rng.uniform(0.5, 1.5, d), dy=rng.standard_normal((T, d))), slot, E


@pytest.mark.parametrize("post", [True, False])
def test_combine_norm_gradients_by_differences(post):
    rng, p, slot, E = problem(1)
    eps, scale, h = 1e-3, 0.7, 1e-6

    def loss(out=p["out"], w=p["w"], go=p["go"]):
        return float(np.sum(p["dy"] * blk.combine_norm(out, slot, w, p["x"], go, post, eps, scale)[0]))
    _, r = blk.combine_norm(p["out"], slot, p["w"], p["x"], p["go"], post, eps, scale)
    dout, dw, dg = blk.combine_norm_backward(p["dy"], p["out"], slot, p["w"], p["go"], post, scale, r)
    for name, grad in (("out", dout), ("w", dw), ("go", dg)):
        for i in np.ndindex(grad.shape):
            e = np.zeros(grad.shape)
            e[i] = h
            diff = (loss(**{name: p[name] + e}) - loss(**{name: p[name] - e})) / (2 * h)
            assert abs(diff - grad[i]) <= 1e-7, (name, i)


def test_dispatch_norm_gradients_by_differences():
    rng, p, slot, E = problem(2)
    eps, h = 1e-3, 1e-6
    T, d = p["x"].shape
    dsend, dg = rng.standard_normal(p["out"].shape), rng.standard_normal((T, E))

    def loss(x=p["x"], gi=p["gi"]):
        """A loss whose gradients with respect to the kept rows of xn, to g and to x itself are dsend, dg and dy."""
        xn, _, g = blk.norm_gate(x, gi, eps, E)
        rows = sum(float(dsend[s] @ xn[m]) for m, s in enumerate(slot) if s >= 0)
        return rows + float(np.sum(dg * g)) + float(np.sum(p["dy"] * x))
    _, r, _ = blk.norm_gate(p["x"], p["gi"], eps, E)
    dx, dgi = blk.dispatch_norm_backward(dsend, slot, dg, p["x"], p["gi"], r, p["dy"])
    for name, grad in (("x", dx), ("gi", dgi)):
        for i in np.ndindex(grad.shape):
            e = np.zeros(grad.shape)
            e[i] = h
            diff = (loss(**{name: p[name] + e}) - loss(**{name: p[name] - e})) / (2 * h)
            assert abs(diff - grad[i]) <= 1e-7, (name, i)


def test_norm_backward_is_reverse_mode():
    rng = np.random.default_rng(3)
    v, dn = torch.tensor(rng.standard_normal((4, 24)), requires_grad=True), torch.tensor(rng.standard_normal((4, 24)))
    (v * (v.square().mean(1, keepdim=True) + 1e-4).rsqrt() * dn).sum().backward()
    n, r = blk.norm(v.detach().numpy(), 1e-4)
    assert np.allclose(blk.norm_backward(dn.numpy(), v.detach().numpy(), r), v.grad.numpy(), rtol=0, atol=1e-13)


def test_layer_few_is_the_layer():
    rng = np.random.default_rng(4)
    T, d, E, h = 9, 12, 3, 8
    x = rng.standard_normal((T, d)).astype(np.float32)
    ws = [(rng.standard_normal((h, d)), rng.standard_normal((d, h))) for _ in range(E)]
    for C in (1, 2, T):
        ref = orc.moe_layer(x, None, np.zeros(E, int), E, 1, C, lambda e: ws[e])
        eid, w, slot, out = blk.layer_few(x, ref["g32"], None, True, C, lambda e: ws[e])
        assert np.array_equal(eid, ref["eid"]) and np.array_equal(slot >= 0, ref["slot"] >= 0)
        assert np.allclose(np.where(slot[:, None] >= 0, w[:, None] * out, 0.0), ref["y"], rtol=0, atol=1e-12)


def test_8_bits():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((7, 40)) * np.exp(rng.standard_normal((7, 1)) * 5)
    z[3, :16] = 0.0
    q, unit = blk.to8(z)
    assert unit.shape == (7, 3) and np.abs(q).max() == 127 and np.array_equal(q, np.round(q))
    back = blk.from8(q, unit)
    # half a unit, and a unit is at most (1 + 2^-8) / 127 of the block's largest value
    for c in range(0, 40, 16):
        most = np.abs(z[:, c:c + 16]).max(axis=1, keepdims=True)
        assert (np.abs(back - z)[:, c:c + 16] <= most * (1 + 2.0 ** -8) / 254 + 1e-300).all()
    # whatever the rounding of the unit does, no value leaves the 8 bits
    for top in np.linspace(1.0, 2.0, 4001):
        assert abs(blk.to8(np.array([[top] + [0.0] * 15]))[0]).max() <= 127
