"""Norms and rotation of queries and keys in 64 bits on the CPU, pairs as complex
numbers, with the gradient written out and magnitudes (the same sums over
absolute values) beside every result."""
import numpy as np


def _split(x, rot, inter):
    z = x[..., :rot]
    return (z[..., 0::2], z[..., 1::2]) if inter else (z[..., :rot // 2], z[..., rot // 2:])


def _join(a, b, rest, inter):
    z = np.stack([a, b], -1).reshape(a.shape[:-1] + (-1,)) if inter else np.concatenate([a, b], -1)
    return np.concatenate([z, rest], -1)


def _turn(y, m, angle, amp, rot, inter, sign):
    """y turned, and its magnitude from m"""
    (a, b), (ma, mb) = _split(y, rot, inter), _split(m, rot, inter)
    z = (a + 1j * b) * np.exp(sign * 1j * angle) * amp
    # an angle off by d moves the pair by d times its length along the circle,
    # whichever component it stands in: the length is both components' magnitude
    size = np.hypot(ma, mb) * abs(amp) * np.ones_like(angle)
    return _join(z.real, z.imag, y[..., rot:], inter), _join(size, size, m[..., rot:], inter)


def rotate(x, w, positions, freq, eps, amp, inter, grad=None):
    """(result, magnitude), and with grad: (dx, m), (dw, m) as well."""
    rot = 2 * len(freq)
    x = np.asarray(x, np.float64)
    angle = np.asarray(positions, np.float64)[..., None, None] * np.asarray(freq, np.float64)
    r, wd = np.ones(x.shape[:-1] + (1,)), np.ones(x.shape[-1])
    if w is not None:
        with np.errstate(divide="ignore"):
            r, wd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps), np.asarray(w, np.float64)
    y = x * r * wd
    got = [_turn(y, np.abs(y), angle, amp, rot, inter, 1)]
    if grad is not None:
        g = np.asarray(grad, np.float64)
        g, mg = _turn(g, np.abs(g), angle, amp, rot, inter, -1)
        if w is None:
            got += [(g, mg), None]
        else:
            gw, mgw = g * wd, mg * np.abs(wd)
            dx = r * gw - x * r ** 3 * (gw * x).mean(-1, keepdims=True)
            mx = r * mgw + np.abs(x) * r ** 3 * (mgw * np.abs(x)).mean(-1, keepdims=True)
            lead = tuple(range(x.ndim - 1))
            got += [(dx, mx), ((g * x * r).sum(lead), (mg * np.abs(x) * r).sum(lead))]
    return got
