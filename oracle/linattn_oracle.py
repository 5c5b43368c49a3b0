"""Plain CPU oracle for linear attention with a decay for each head.

TEST INFRASTRUCTURE ONLY (see made_oracle.py for the rules; nothing in the product path imports this).

One sequence, fp64, one step after the other, exactly as the recurrence is written:

    S_t = lambda S_{t-1} + k_t v_t^T,     o_t = scale S_t^T q_t,     lambda = exp(log_decay)

q [T, heads, Dk], k [T, kv_heads, Dk], v [T, kv_heads, Dv], log_decay [kv_heads], states [kv_heads, Dk, Dv]; query head h
reads state h // (heads // kv_heads).  The gradients follow by going through the steps backwards with dS_t = dL/dS_t:

    dS_t = lambda dS_{t+1} + scale sum_h q_t^h (do_t^h)^T      (heads h of the state; dS_T also gets d_state_out)
    dq_t^h = scale S_t do_t^h,   dk_t = dS_t v_t,   dv_t = dS_t^T k_t,   d_state_in = lambda dS_1
"""
from __future__ import annotations

import numpy as np


def forward(q, k, v, log_decay, scale, state=None):
    """-> (o [T, heads, Dv], last state, states [T, kv_heads, Dk, Dv] after every step)"""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, heads, Dk = q.shape
    n, Dv = v.shape[1:]
    G = heads // n
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((n, Dk, Dv)) if state is None else np.array(state, np.float64)
    o, states = np.zeros((T, heads, Dv)), np.zeros((T, n, Dk, Dv))
    for t in range(T):
        S = lam * S + k[t][:, :, None] * v[t][:, None, :]
        states[t] = S
        for h in range(heads):
            o[t, h] = scale * (S[h // G].T @ q[t, h])
    return o, S, states


def backward(q, k, v, log_decay, scale, do, state=None, d_state_out=None):
    """-> (dq, dk, dv, d_state_in)"""
    q, k, v, do = (np.asarray(x, np.float64) for x in (q, k, v, do))
    T, heads, Dk = q.shape
    n, Dv = v.shape[1:]
    G = heads // n
    _, _, states = forward(q, k, v, log_decay, scale, state)
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    dS = np.zeros((n, Dk, Dv)) if d_state_out is None else np.array(d_state_out, np.float64)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for t in range(T - 1, -1, -1):
        for h in range(heads):
            dS[h // G] += scale * np.outer(q[t, h], do[t, h])
            dq[t, h] = scale * (states[t, h // G] @ do[t, h])
        for h in range(n):
            dk[t, h] = dS[h] @ v[t, h]
            dv[t, h] = dS[h].T @ k[t, h]
        dS = lam * dS
    return dq, dk, dv, dS
