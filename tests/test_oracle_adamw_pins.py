"""Pins of oracle/adamw_oracle.py (CPU only): closed forms of the step and properties of the 8-bit codes."""
import numpy as np
import torch

from oracle import adamw_oracle as A


def test_first_step_moves_by_lr_against_the_gradient():
    p, m, v = A.step([1.0, -2.0], [0.5, -3.0], [0, 0], [0, 0], 0.1, 0.9, 0.999, 0.0, 0.0, 1)
    assert np.allclose(p, [0.9, -1.9]) and np.allclose(m, [0.05, -0.3]) and np.allclose(v, [0.00025, 0.009])


def test_weight_decay_alone():
    p, _, _ = A.step([4.0], [0.0], [0.0], [0.0], 0.1, 0.9, 0.99, 1e-8, 0.5, 3)
    assert np.allclose(p, [4.0 * 0.95])


def test_ten_steps_against_torch():
    g = np.random.default_rng(0)
    w = torch.tensor(g.normal(size=50), dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([w], lr=0.02, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    p, m, v = w.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 11):
        grad = g.normal(size=50)
        w.grad = torch.tensor(grad)
        opt.step()
        p, m, v = A.step(p, grad, m, v, 0.02, 0.8, 0.95, 1e-6, 0.1, t)
    assert np.abs(p - w.detach().numpy()).max() < 1e-14


def test_codes_are_nearest_in_their_roots():
    g = np.random.default_rng(1)
    m, v = g.normal(size=1000) * np.exp(g.normal(size=1000) * 3), np.exp(g.normal(size=1000) * 5)
    m[3], v[5] = 0.0, 0.0
    mc, vc, ms, vs = A.pack(m, v)
    mu, vu = A.unpack(mc, vc, ms, vs)
    at = np.arange(1000) // 256
    # half a step of the root, and 2^-24 for the scale's rounding
    assert (np.abs(np.sqrt(np.abs(mu / ms[at])) - np.sqrt(np.abs(m / ms[at]))) <= 0.5 / 127 + 1e-6).all()
    err = np.abs((vu / vs[at]) ** 0.25 - (v / vs[at]) ** 0.25)
    assert (err <= np.where(vc == 1, 1.0, 0.5) / 255 + 1e-6).all()
    assert mc[3] == 0 and vc[5] == 0 and (vc[v > 0] >= 1).all() and (np.sign(mu) * np.sign(m) >= 0).all()


def test_values_have_their_own_codes():
    mc = np.arange(-127, 129).clip(-127, 127).astype(np.int8)
    vc = np.arange(256).astype(np.uint8)
    mu, vu = A.unpack(mc, vc, [3.0], [5.0])
    m2, v2, ms, vs = A.pack(mu, vu)
    assert (m2 == mc).all() and (v2 == vc).all() and ms[0] == 3 and vs[0] == 5
