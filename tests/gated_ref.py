"""The gated recurrence and its gradient in 64 bits on the CPU, step by step, with
magnitudes (the same sums over absolute values) beside every result; and dropout's
random numbers in Python integers."""
import numpy as np


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(v, np.float64)))


def gates_of(gates, alpha):
    r, i = np.asarray(gates[..., 0, :], np.float64), np.asarray(gates[..., 1, :], np.float64)
    u = np.abs(np.asarray(alpha, np.float64)) * sigmoid(r)
    return dict(u=u, a=np.exp(-u), m=np.sqrt(-np.expm1(-2.0 * u)), si=sigmoid(i), sr=sigmoid(r), ci=sigmoid(-i), cr=sigmoid(-r))


def scan(x, gates, alpha, start, state=None):
    """h [B,T,d] and its magnitude, the state after the last step and its magnitude."""
    g = gates_of(gates, alpha)
    b = g["m"] * g["si"] * np.asarray(x, np.float64)
    B, T, d = b.shape
    now = np.zeros((B, d)) if state is None else np.asarray(state, np.float64).copy()
    mag = np.abs(now)
    h, m = np.empty_like(b), np.empty_like(b)
    for t in range(T):
        on = np.asarray(start[:, t] == 0)[:, None]
        now = np.where(on, g["a"][:, t] * now, 0.0) + b[:, t]
        mag = np.where(on, g["a"][:, t] * mag, 0.0) + np.abs(b[:, t])
        h[:, t], m[:, t] = now, mag
    return h, m, now, mag


def grads(x, gates, alpha, start, grad_h, state=None, grad_state=None):
    """{name: (gradient, magnitude)} of x, gates, alpha and the state.  1 - sigmoid is a
    difference in the kernels: where its relative error is that of 1, the magnitude
    has 1 in its place."""
    x = np.asarray(x, np.float64)
    h, mh, _, _ = scan(x, gates, alpha, start, state)
    g = gates_of(gates, alpha)
    B, T, d = x.shape
    s0 = np.zeros((B, d)) if state is None else np.asarray(state, np.float64)
    c = np.zeros((B, d)) if grad_state is None else np.asarray(grad_state, np.float64)
    mc = np.abs(c)
    dx, dr, di = (np.empty_like(x) for _ in range(3))
    mx, mr, mi = (np.empty_like(x) for _ in range(3))
    da, ma = np.zeros(d), np.zeros(d)
    for t in range(T - 1, -1, -1):
        on = np.asarray(start[:, t] == 0)[:, None]
        a, m, si, sr, u, ci, cr = (g[k][:, t] for k in ("a", "m", "si", "sr", "u", "ci", "cr"))
        lam = np.asarray(grad_h[:, t], np.float64) + c
        ml = np.abs(np.asarray(grad_h[:, t], np.float64)) + mc
        before, mb = (h[:, t - 1], mh[:, t - 1]) if t else (s0, np.abs(s0))
        before, mb = np.where(on, before, 0.0), np.where(on, mb, 0.0)
        with np.errstate(divide="ignore", invalid="ignore"):
            am = np.where(m > 0, a / np.where(m > 0, m, 1.0), 0.0)
        b = m * si * x[:, t]
        du, mu = lam * a * (si * x[:, t] * am - before), ml * a * (si * np.abs(x[:, t]) * am + mb)
        dx[:, t], mx[:, t] = lam * m * si, ml * m * si
        di[:, t], mi[:, t] = lam * b * ci, ml * np.abs(b)
        dr[:, t], mr[:, t] = du * u * cr, mu * u
        da += (du * sr).sum(0)
        ma += (mu * sr).sum(0)
        c, mc = np.where(on, a * lam, 0.0), np.where(on, a * ml, 0.0)
    sign = np.sign(np.asarray(alpha, np.float64))
    return {"x": (dx, mx), "gates": (np.stack([dr, di], 2), np.stack([mr, mi], 2)), "alpha": (sign * da, np.abs(sign) * ma),
            "state": (c, mc)}


# ------------------------------------------------------------------ dropout

def philox(counter, key):
    """Philox4x32-10 on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def numbers(seed, step, site, rows, d, first_row=0):
    """The 32-bit numbers of elements [first_row ..][d]."""
    seed, step = seed % (1 << 64), step % (1 << 32)
    out = np.empty((rows, d), np.uint64)
    for i in range(rows):
        for block in range((d + 7) // 8):
            halves = []
            for top in (0, 1 << 31):
                w = philox([block | top, first_row + i, step, site], [seed & 0xFFFFFFFF, seed >> 32])
                halves.append([v for x in w for v in (x & 0xFFFF, x >> 16)])
            for e in range(min(8, d - 8 * block)):
                out[i, 8 * block + e] = (halves[0][e] << 16) | halves[1][e]
    return out


def keep(p, seed, step, site, rows, d, first_row=0):
    return numbers(seed, step, site, rows, d, first_row) >= np.uint64(round(p * 2.0 ** 32))


# --------------------------------------------------------------- layer norm

def norm(s, w, b, eps, ms=None):
    """y and its magnitude for rows s (whose own magnitude is ms)."""
    s = np.asarray(s, np.float64)
    ms = np.abs(s) if ms is None else ms
    mean = s.mean(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt(((s - mean) ** 2).mean(-1, keepdims=True) + eps)
    w = np.ones(s.shape[-1]) if w is None else np.asarray(w, np.float64)
    b = np.zeros(s.shape[-1]) if b is None else np.asarray(b, np.float64)
    return (s - mean) * r * w + b, (ms + ms.mean(-1, keepdims=True)) * r * np.abs(w) + np.abs(b), mean, r


def norm_grads(s, w, eps, gy, gs=None):
    """ds, dw, db, each with its magnitude."""
    s, gy = np.asarray(s, np.float64), np.asarray(gy, np.float64)
    _, _, mean, r = norm(s, w, None, eps)
    w = np.ones(s.shape[-1]) if w is None else np.asarray(w, np.float64)
    xh, mxh = (s - mean) * r, (np.abs(s) + np.abs(s).mean(-1, keepdims=True)) * r
    gw, mg = gy * w, np.abs(gy * w)
    ds = r * (gw - gw.mean(-1, keepdims=True) - xh * (gw * xh).mean(-1, keepdims=True))
    # (rstd's relative error goes into every term; xh's into both of its places)
    ms = r * (mg + mg.mean(-1, keepdims=True) + mxh * (mg * mxh).mean(-1, keepdims=True))
    if gs is not None:
        ds, ms = ds + np.asarray(gs, np.float64), ms + np.abs(np.asarray(gs, np.float64))
    lead = tuple(range(s.ndim - 1))
    return (ds, ms), ((gy * xh).sum(lead), (np.abs(gy) * mxh).sum(lead)), (gy.sum(lead), np.abs(gy).sum(lead))
