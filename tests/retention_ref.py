"""Retention in 64 bits, step by step on the CPU: the recurrence and its
derivative written out, with nothing in common with the kernels' chunks."""
import numpy as np


def share(x, H):
    """[B,T,Hk,d] -> [B,T,H,d]: the key heads repeated for their query heads."""
    return np.repeat(x, H // x.shape[2], axis=2)


def forward(q, k, v, alpha, start, scale, state=None):
    """(out, state after the last step, every state S_t)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, T, H, dk = q.shape
    k, v = share(k, H), share(v, H)
    gamma = np.exp(-np.abs(np.asarray(alpha, np.float64)))[None, :, None, None]
    S = np.zeros((B, H, dk, v.shape[3])) if state is None else np.asarray(state, np.float64).copy()
    out = np.zeros((B, T, H, v.shape[3]))
    states = np.zeros((T,) + S.shape)
    for t in range(T):
        begins = (start[:, t] != 0)[:, None, None, None]
        S = np.where(begins, 0.0, gamma * S) + k[:, t, :, :, None] * v[:, t, :, None, :]
        out[:, t] = scale * (q[:, t, :, :, None] * S).sum(2)
        states[t] = S
    return out, S, states


def backward(q, k, v, alpha, start, scale, grad_out, state=None, grad_state=None):
    """dict of dq, dk, dv, dalpha, dstate."""
    q, k, v, g = (np.asarray(x, np.float64) for x in (q, k, v, grad_out))
    B, T, H, dk = q.shape
    Hk, dv = v.shape[2:]
    states = forward(q, k, v, alpha, start, scale, state)[2]
    first = np.zeros(states.shape[1:]) if state is None else np.asarray(state, np.float64)
    kh, vh = share(k, H), share(v, H)
    a = np.asarray(alpha, np.float64)
    gamma = np.exp(-np.abs(a))[None, :, None, None]
    dS = np.zeros_like(first) if grad_state is None else np.asarray(grad_state, np.float64).copy()
    dq, dkk, dvv, dlog = np.zeros(q.shape), np.zeros((B, T, H, dk)), np.zeros((B, T, H, dv)), np.zeros(H)
    for t in range(T - 1, -1, -1):
        dS = dS + scale * q[:, t, :, :, None] * g[:, t, :, None, :]
        dq[:, t] = scale * (states[t] * g[:, t, :, None, :]).sum(3)
        dkk[:, t] = (dS * vh[:, t, :, None, :]).sum(3)
        dvv[:, t] = (dS * kh[:, t, :, :, None]).sum(2)
        begins = (start[:, t] != 0)[:, None, None, None]
        before = states[t - 1] if t else first
        dlog += np.where(begins, 0.0, gamma * before * dS).sum((0, 2, 3))
        dS = np.where(begins, 0.0, gamma * dS)
    G = H // Hk
    return dict(dq=dq, dk=dkk.reshape(B, T, Hk, G, dk).sum(3), dv=dvv.reshape(B, T, Hk, G, dv).sum(3),
                dalpha=-np.sign(a) * dlog, dstate=dS)


def magnitudes(q, k, v, alpha, start, scale, grad_out=None, state=None, grad_state=None):
    """The same sums over absolute values: what a rounding error scales with."""
    ab = [None if x is None else np.abs(np.asarray(x, np.float64)) for x in (q, k, v, grad_out, state, grad_state)]
    q, k, v, grad_out, state, grad_state = ab
    out, S, _ = forward(q, k, v, alpha, start, abs(scale), state)
    m = dict(out=out, state=S)
    if grad_out is not None:
        b = backward(q, k, v, alpha, start, abs(scale), grad_out, state, grad_state)
        b["dalpha"] = np.abs(b["dalpha"])
        m.update(b)
    return m
