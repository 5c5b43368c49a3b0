"""Pins of oracle/linattn_oracle.py (CPU only): closed forms of the recurrence, and its gradients against differences."""
import numpy as np
import pytest

from oracle import linattn_oracle as L


def draw(T, heads, kv, Dk, Dv, seed=0):
    g = np.random.default_rng(seed)
    return (g.normal(size=(T, heads, Dk)), g.normal(size=(T, kv, Dk)), g.normal(size=(T, kv, Dv)),
            -g.uniform(0.01, 1.0, size=kv), g.normal(size=(kv, Dk, Dv)), g.normal(size=(T, heads, Dv)), g.normal(size=(kv, Dk, Dv)))


def test_no_decay_is_attention_without_its_softmax():
    q, k, v, _, _, _, _ = draw(11, 2, 2, 5, 3)
    o = L.forward(q, k, v, np.zeros(2), 0.7)[0]
    for h in range(2):
        scores = np.tril(q[:, h] @ k[:, h].T)
        assert np.allclose(o[:, h], 0.7 * scores @ v[:, h], atol=1e-12)


def test_no_memory_sees_its_own_step_alone():
    q, k, v, _, s, _, _ = draw(6, 1, 1, 4, 3)
    o, end, _ = L.forward(q, k, v, np.array([-np.inf]), 1.0, s)
    assert np.allclose(o[:, 0], (q[:, 0] * k[:, 0]).sum(1, keepdims=True) * v[:, 0], atol=1e-12)
    assert np.allclose(end[0], np.outer(k[-1, 0], v[-1, 0]))


def test_a_sequence_in_two_parts_and_without_steps():
    q, k, v, ld, s, _, _ = draw(9, 4, 2, 5, 3)
    o, end, _ = L.forward(q, k, v, ld, 0.3, s)
    o1, mid, _ = L.forward(q[:4], k[:4], v[:4], ld, 0.3, s)
    o2, end2, _ = L.forward(q[4:], k[4:], v[4:], ld, 0.3, mid)
    assert np.allclose(np.concatenate([o1, o2]), o) and np.allclose(end, end2)
    none = L.forward(q[:0], k[:0], v[:0], ld, 0.3, s)
    assert none[0].shape == (0, 4, 3) and (none[1] == s).all()


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 2), (3, 1)])
def test_gradients_against_differences(heads, kv):
    q, k, v, ld, s, do, ds = draw(7, heads, kv, 4, 3, seed=heads)

    def loss(q, k, v, s):
        o, end, _ = L.forward(q, k, v, ld, 0.4, s)
        return (o * do).sum() + (end * ds).sum()

    grads = L.backward(q, k, v, ld, 0.4, do, s, ds)
    args = [q, k, v, s]
    for i, g in enumerate(grads):
        num = np.zeros_like(args[i])
        for at in np.ndindex(num.shape):
            hi, lo = [x.copy() for x in args], [x.copy() for x in args]
            hi[i][at] += 1e-5
            lo[i][at] -= 1e-5
            num[at] = (loss(*hi) - loss(*lo)) / 2e-5
        assert np.abs(g - num).max() < 1e-7
