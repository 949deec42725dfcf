"""The retention operators -- linear attention whose state decays at a rate of
its own in each head -- with what prepares their queries and keys: the cases
they are timed on, their plain forms and their 64-bit results.

Per head, over a tape of episodes, with gamma = exp(-|alpha|),

    S_t = gamma S_{t-1} + k_t^T v_t      (S_t = k_t^T v_t where an episode begins)
    out_t = scale q_t S_t

``kind`` says which operator a case runs, each through the torch layer of
``paper_2402_09900_amd.binding``:

* ``scan``: a whole tape at once, from a carried state on if there is one, and
  the state after it: evaluating rollouts, reading a prompt;
* ``train``: the same through autograd, with the gradients of q, k, v, the
  decay rates and the carried state;
* ``step``: one step of every environment or sequence, the state updated in
  place: acting, generating;
* ``rotate``: RMS norms of queries and keys per head and the position rotation;
* ``rotate_train``: the same through autograd, with the gradients of q, k and
  the norms' weights.

The inputs are drawn on the GPU from a seed: normal q, k, v, rates spread over
their logarithm from 1/8 (a memory of a few steps) to 1/4096, episode lengths
with the laws of ``paper_2402_09900_amd.tapes``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ------------------------------------------------------------------- cases

def _ret(kind, dtype, B, T, H, Hk, dk, dv, carry, mean, **more):
    return dict(kind=kind, dtype=dtype, B=B, T=T, H=H, Hk=Hk, dk=dk, dv=dv, carry=carry, mean=float(mean), **more)


def _rot(kind, dtype, B, T, H, Hk, d, rot, interleaved, norm, far):
    return dict(kind=kind, dtype=dtype, B=B, T=T, H=H, Hk=Hk, d=d, rot=rot, interleaved=interleaved, norm=norm, far=far)


def listed():
    return [
        # acting in 16 environments, the linear-attention layer's usual 4 heads
        # of 64: the smallest call, latency counts
        dict(_ret("step", "f32", 16, 1, 4, 4, 64, 64, True, 100), name="step_f32_B16_H4_d64"),
        # generating for 256 sequences, 16 heads of 128: 1 MiB of state a sequence
        dict(_ret("step", "bf16", 256, 1, 16, 16, 128, 128, True, 500), name="step_bf16_B256_H16_d128"),
        # evaluating one short rollout, with the state to go on from
        dict(_ret("scan", "f32", 1, 1000, 4, 4, 64, 64, True, 100), name="scan_f32_T1000_H4_d64"),
        # reading one long prompt
        dict(_ret("scan", "bf16", 1, 65536, 16, 16, 128, 128, True, 20000), name="scan_bf16_T65536_H16_d128"),
        # training on a Tape-Based batch: the linear-attention workload's size
        dict(_ret("train", "f32", 1, 32768, 4, 4, 64, 64, False, 500), name="train_f32_T32768_H4_d64"),
        # training on eight rows of packed sequences
        dict(_ret("train", "bf16", 8, 4096, 16, 16, 128, 128, False, 1500), name="train_bf16_B8_T4096_H16_d128"),
        # ragged: shared keys and values, head widths that fill no tile, a length
        # that fills no chunk, truncated episodes going on from a carried state
        dict(_ret("train", "bf16", 3, 1999, 6, 2, 80, 96, True, 300), name="train_bf16_B3_T1999_H6_2_d80_96"),
        # one long sequence of 32 query heads on 8 key heads: the largest
        dict(_ret("train", "bf16", 1, 32768, 32, 8, 128, 128, True, 9000), name="train_bf16_T32768_H32_8_d128"),
        # queries and keys of one token for each of 64 sequences at far positions
        dict(_rot("rotate", "bf16", 64, 1, 16, 16, 128, 128, False, True, 1 << 17), name="rotate_bf16_B64_T1_H16_d128"),
        # queries and keys of the long prompt
        dict(_rot("rotate", "bf16", 1, 65536, 16, 16, 128, 128, False, True, 0), name="rotate_bf16_T65536_H16_d128"),
        # training, ragged: a quarter of the head turned, neighbours as pairs
        dict(_rot("rotate_train", "f32", 3, 1999, 6, 2, 80, 20, True, True, 0), name="rotate_train_f32_B3_T1999_d80"),
        # training on the long sequence
        dict(_rot("rotate_train", "bf16", 1, 32768, 32, 8, 128, 64, False, True, 0),
             name="rotate_train_bf16_T32768_H32_8_d128"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "scan", "scan", "train", "train", "train", "rotate", "rotate_train"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    Hk = rng.choice([1, 2, 3, 4, 4, 8, 16])
    H = Hk * rng.choice([1, 1, 1, 2, 4])
    if kind.startswith("rotate"):
        d = rng.choice([32, 64, 64, 80, 96, 128, 128])
        rot = rng.choice([d, d, d // 2, d // 4])
        B = _logint(rng, 1, 64)
        total = _logint(rng, 1 << 14, 1 << 26)
        return _rot(kind, dtype, B, max(1, total // (B * (H + Hk) * d)), H, Hk, d, rot, rng.random() < 0.4,
                    rng.random() < 0.75, rng.choice([0, 1 << 17]))
    dk = rng.choice([32, 64, 64, 80, 96, 128, 128])
    dv = rng.choice([dk, dk, 64, 128, 40])
    mean = _logint(rng, 20, 20000)
    if kind == "step":
        return _ret(kind, dtype, max(1, _logint(rng, 1 << 14, 1 << 26) // (H * dk * dv)), 1, H, Hk, dk, dv, True, mean)
    # up to 2^26 values of v, and up to 2^14 (head, chunk of 64 rows) pairs for f32
    total = _logint(rng, 1 << 14, 1 << (26 if dtype == "bf16" else 24))
    B = _logint(rng, 1, 16)
    return _ret(kind, dtype, B, min(65536, max(64, total // (B * H * max(dk, dv))) + rng.randrange(16)), H, Hk, dk, dv,
                rng.random() < 0.5, mean)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, dtype, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _flags(case, rng):
    """Begin flags of B tapes laid end to end and cut: a tape of a carried state
    may start inside an episode."""
    B, T = case["B"], case["T"]
    f = np.zeros(B * T, np.uint8)
    at = 0 if not case["carry"] else int(rng.integers(0, max(1, int(case["mean"]))))
    while at < B * T:
        f[at] = 1
        at += int(rng.geometric(1.0 / case["mean"]))
    f = f.reshape(B, T)
    if not case["carry"]:
        f[:, 0] = 1
    return torch.from_numpy(f).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    dt = DTYPES[case["dtype"]]
    B, T, H, Hk = case["B"], case["T"], case["H"], case["Hk"]
    s = {"case": case}
    if case["kind"].startswith("rotate"):
        d, rot = case["d"], case["rot"]
        s["q"] = _normal(g, dt, B, T, H, d)
        s["k"] = _normal(g, dt, B, T, Hk, d)
        first = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device=DEV)
        s["positions"] = (first + torch.arange(T, device=DEV)).to(torch.int32)
        s["freq"] = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)).float()
        s["wq"] = 1.0 + 0.1 * _normal(g, torch.float32, d) if case["norm"] else None
        s["wk"] = 1.0 + 0.1 * _normal(g, torch.float32, d) if case["norm"] else None
        if case["kind"] == "rotate_train":
            s["gq"], s["gk"] = _normal(g, dt, B, T, H, d), _normal(g, dt, B, T, Hk, d)
        return s
    dk, dv = case["dk"], case["dv"]
    step = case["kind"] == "step"
    lead = (B,) if step else (B, T)
    s["q"] = _normal(g, dt, *lead, H, dk)
    s["k"] = _normal(g, dt, *lead, Hk, dk)
    s["v"] = _normal(g, dt, *lead, Hk, dv)
    # rates from 1/8 to 1/4096, log-spaced over the heads and jittered; the sign
    # of alpha means nothing
    u = (torch.arange(H, device=DEV) + torch.rand(H, generator=g, device=DEV)) / H
    s["alpha"] = torch.exp(-math.log(8.0) - u * math.log(512.0)) * (1.0 - 2.0 * (torch.arange(H, device=DEV) % 2))
    s["scale"] = dk ** -0.5
    rng = np.random.Generator(np.random.PCG64(int(seed)))
    if step:
        s["start"] = (torch.rand(B, generator=g, device=DEV) < 1.0 / case["mean"]).to(torch.uint8)
    else:
        s["start"] = _flags(case, rng)
    s["state"] = _normal(g, torch.float32, B, H, dk, dv) if case["carry"] else None
    if case["kind"] == "train":
        s["grad_out"] = _normal(g, dt, B, T, H, dv)
        s["grad_state"] = _normal(g, torch.float32, B, H, dk, dv) if case["carry"] else None
    return s


# -------------------------------------------------------------- plain forms

_ROWS = 256                 # rows of a block in the plain form


def _shared(x, H):
    """The key heads repeated for the query heads that share them."""
    return x.repeat_interleave(H // x.shape[-2], dim=-2) if x.shape[-2] != H else x


def _blocks(x, N, C):
    """[B, T, H, d] as [B, H, N, C, d], zeros behind the tape's end."""
    B, T, H, d = x.shape
    x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, N * C - T))
    return x.reshape(B, N, C, H, d).permute(0, 3, 1, 2, 4).contiguous()


def _decays(alpha, steps):
    """gamma^steps per head, its exponent in 64 bits (32 lose the slow rates)."""
    rate = alpha.double().abs()
    return torch.exp(-rate.reshape((-1,) + (1,) * steps.dim()) * steps.double()).float()


def _plain_scan(q, k, v, alpha, start, scale, state):
    """The scan in blocks of C rows: the rows of a block against each other, the
    states that the blocks add, and the rows against the state before them.
    Returns out (32 bits) and the state after the last step."""
    B, T, H, dk = q.shape
    dv = v.shape[3]
    C = min(_ROWS, T)
    N = -(-T // C)
    dev = q.device
    qb, kb, vb = _blocks(q, N, C), _blocks(_shared(k.float(), H), N, C), _blocks(_shared(v.float(), H), N, C)
    # episode of each row, 0 = the one that the carried state belongs to
    ep = torch.nn.functional.pad(torch.cumsum((start != 0).long(), 1), (0, N * C - T), value=-1).reshape(B, N, C)
    i = torch.arange(C, device=dev)
    n = torch.arange(N, device=dev)
    # rows of a block against each other
    seen = (ep[:, :, :, None] == ep[:, :, None, :]) & (i[:, None] >= i[None, :])            # [B, N, C, C]
    near = _decays(alpha, (i[:, None] - i[None, :]).clamp(min=0))[None, :, None]            # [1, H, 1, C, C]
    p = torch.matmul(qb, kb.transpose(-1, -2)) * near * seen[:, None]
    out = torch.matmul(p, vb)
    # what each block adds to the state after its last valid row
    rows = (T - n * C).clamp(max=C)                                                         # [N]
    last = ep.gather(2, (rows - 1)[None, :, None].expand(B, N, 1))                          # [B, N, 1]
    w = _decays(alpha, (rows[:, None] - 1 - i[None, :]).clamp(min=0))[None]                 # [1, H, N, C]
    w = w * (ep == last)[:, None]
    add = torch.matmul((kb * w[..., None]).transpose(-1, -2), vb).reshape(B, H, N, dk * dv)
    # the state before each block and after the last, from what the blocks added
    # and the carried state in place -1
    m = torch.arange(N + 1, device=dev)
    ends = torch.minimum(m * C, torch.tensor(T, device=dev))                                # steps before block m
    ids = torch.cat([torch.zeros(B, 1, device=dev, dtype=ep.dtype), last[:, :, 0]], 1)      # [B, N + 1]
    far = _decays(alpha, (ends[:, None] - ends[None, :]).clamp(min=0))                      # [H, N + 1, N + 1]
    keep = (ids[:, :, None] == ids[:, None, :]) & (m[:, None] >= m[None, :])
    first = torch.zeros(B, H, 1, dk * dv, device=dev) if state is None else state.float().reshape(B, H, 1, dk * dv)
    states = torch.matmul(far[None] * keep[:, None], torch.cat([first, add], 2))            # [B, H, N + 1, dk dv]
    goes_on = (ep == ids[:, :N, None])[:, None] * _decays(alpha, i + 1)[None, :, None, :]   # [B, H, N, C]
    out = out + torch.matmul(qb, states[:, :, :N].reshape(B, H, N, dk, dv)) * goes_on[..., None]
    out = (out * scale).permute(0, 2, 3, 1, 4).reshape(B, N * C, H, dv)[:, :T]
    return out, states[:, :, N].reshape(B, H, dk, dv)


def _plain_step(s):
    c = s["case"]
    q, k, v = s["q"].float(), _shared(s["k"].float(), c["H"]), _shared(s["v"].float(), c["H"])
    goes_on = (s["start"] == 0).float()[:, None, None, None]
    gamma = torch.exp(-s["alpha"].double().abs()).float()[None, :, None, None]
    new = s["state"] * (gamma * goes_on) + k[..., :, None] * v[..., None, :]
    s["state"].copy_(new)
    return {"out": (torch.matmul(q[..., None, :], new)[..., 0, :] * s["scale"]).to(s["q"].dtype), "state": s["state"]}


def _plain_rotate(x, w, s):
    c = s["case"]
    rot, d = c["rot"], c["d"]
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    angle = s["positions"].double()[..., None, None] * s["freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1) if rot < d else turned


def _leaves(*tensors):
    return [None if t is None else t.detach().requires_grad_(True) for t in tensors]


def _grads(outs, grads, leaves, names):
    got = torch.autograd.grad([o for o, g in zip(outs, grads) if g is not None], [x for x in leaves if x is not None],
                              [g for g in grads if g is not None])
    got = list(got)
    return {n: got.pop(0) for n, x in zip(names, leaves) if x is not None}


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        return _run_own(s, c, kind)
    if kind == "step":
        return _plain_step(s)
    dt = s["q"].dtype
    if kind == "scan":
        out, state = _plain_scan(s["q"], s["k"], s["v"], s["alpha"], s["start"], s["scale"], s["state"])
        return {"out": out.to(dt), "state": state}
    if kind == "train":
        leaves = _leaves(s["q"], s["k"], s["v"], s["alpha"], s["state"])
        out, state = _plain_scan(*leaves[:4], s["start"], s["scale"], leaves[4])
        out = out.to(dt)
        r = _grads((out, state), (s["grad_out"], s["grad_state"]), leaves, ("dq", "dk", "dv", "dalpha", "dstate"))
        return {"out": out.detach(), **r}
    if kind == "rotate":
        return {"q": _plain_rotate(s["q"], s["wq"], s).to(dt), "k": _plain_rotate(s["k"], s["wk"], s).to(dt)}
    leaves = _leaves(s["q"], s["k"], s["wq"], s["wk"])
    q, k = _plain_rotate(leaves[0], leaves[2], s).to(dt), _plain_rotate(leaves[1], leaves[3], s).to(dt)
    r = _grads((q, k), (s["gq"], s["gk"]), leaves, ("dq", "dk", "dwq", "dwk"))
    return {"q": q.detach(), "k": k.detach(), **r}


# ------------------------------------------------------ the framework's calls

def _run_own(s, c, kind):
    from paper_2402_09900_amd import binding as mb
    if kind == "step":
        out = mb.retention_step(s["q"], s["k"], s["v"], s["alpha"], s["state"], s["start"], scale=s["scale"])
        return {"out": out, "state": s["state"]}
    if kind == "scan":
        out, state = mb.scan_retention(s["q"], s["k"], s["v"], s["alpha"], s["start"], scale=s["scale"],
                                       state=s["state"], final_state=True)
        return {"out": out, "state": state}
    if kind == "train":
        leaves = _leaves(s["q"], s["k"], s["v"], s["alpha"], s["state"])
        got = mb.retention(*leaves[:4], s["start"], scale=s["scale"], state=leaves[4],
                           final_state=s["grad_state"] is not None)
        out, state = got if s["grad_state"] is not None else (got, None)
        r = _grads((out, state), (s["grad_out"], s["grad_state"]), leaves, ("dq", "dk", "dv", "dalpha", "dstate"))
        return {"out": out.detach(), **r}
    if kind == "rotate":
        q, k = mb.rotate_qk(s["q"], s["k"], s["positions"], s["freq"], wq=s["wq"], wk=s["wk"], eps=EPS,
                            interleaved=c["interleaved"])
        return {"q": q, "k": k}
    leaves = _leaves(s["q"], s["k"], s["wq"], s["wk"])
    q, k = mb.qk_rotate(leaves[0], leaves[1], s["positions"], s["freq"], wq=leaves[2], wk=leaves[3], eps=EPS,
                        interleaved=c["interleaved"])
    r = _grads((q, k), (s["gq"], s["gk"]), leaves, ("dq", "dk", "dwq", "dwk"))
    return {"q": q.detach(), "k": k.detach(), **r}


# --------------------------------------------------------------------- work

def work(case):
    """Bytes: each input once, each output once.  Flops of a scan: a row against
    the state (2 dk dv) and into it (2 dk dv); of its gradient, the same for each
    of dq, dk, dv and twice over for the decay rates (the state and its
    derivative by the rate).  Chunked forms do more; none is needed."""
    e = 4 if case["dtype"] == "f32" else 2
    B, T, H, Hk = case["B"], case["T"], case["H"], case["Hk"]
    n = B * T
    if case["kind"].startswith("rotate"):
        x = n * (H + Hk) * case["d"]
        small = 4 * n + 2 * case["rot"] + (8 * case["d"] if case["norm"] else 0)
        if case["kind"] == "rotate":
            return {"bytes": 2.0 * x * e + small, "flops": 10.0 * x}
        return {"bytes": 4.0 * x * e + 2.0 * small, "flops": 30.0 * x}
    dk, dv = case["dk"], case["dv"]
    ins = n * (H * dk + Hk * (dk + dv)) * e + n + 4 * H
    outs = n * H * dv * e
    st = 4 * B * H * dk * dv
    fwd = 4.0 * n * H * dk * dv
    if case["kind"] == "step":
        return {"bytes": float(ins + outs + 2 * st), "flops": fwd + 1.0 * n * H * dk * dv}
    if case["kind"] == "scan":
        return {"bytes": float(ins + outs + (2 if case["carry"] else 1) * st), "flops": fwd}
    # the inputs, grad_out in; out and the gradients out; with a carried state: it,
    # its gradient and the gradient of the one after the tape
    return {"bytes": float(2 * ins + 2 * outs + (3 if case["carry"] else 0) * st), "flops": 6 * fwd}


# -------------------------------------------------------------------- 64 bits

def _exact_scan(s, grads):
    """Rows against all earlier rows of their episode, in 64 bits: weights
    gamma^(i - j) over pairs, a block of query rows at a time."""
    c = s["case"]
    B, T, H, Hk, dk, dv = (c[x] for x in ("B", "T", "H", "Hk", "dk", "dv"))
    G, scale, carry = H // Hk, s["scale"], s["state"] is not None
    out = torch.zeros(B, T, H, dv, dtype=torch.float64, device=DEV)
    state = torch.zeros(B, H, dk, dv, dtype=torch.float64, device=DEV)
    if grads:
        dq = torch.zeros(B, T, H, dk, dtype=torch.float64, device=DEV)
        dkk = torch.zeros(B, T, Hk, dk, dtype=torch.float64, device=DEV)
        dvv = torch.zeros(B, T, Hk, dv, dtype=torch.float64, device=DEV)
        dlog = torch.zeros(H, dtype=torch.float64, device=DEV)
        dstate = torch.zeros(B, H, dk, dv, dtype=torch.float64, device=DEV)
    R = 1024
    for b in range(B):
        begin = torch.nonzero(s["start"][b]).flatten().cpu().numpy()
        # first step of each step's episode; -1: the carried state's episode
        begins = np.full(T, -1, np.int64)
        begins[begin] = begin
        begins = np.maximum.accumulate(begins)
        ep = torch.from_numpy(begins).to(DEV)
        for h in range(H):
            kh = h // G
            rate = float(s["alpha"][h].double().abs())
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :, kh].double(), s["v"][b, :, kh].double()
            s0 = s["state"][b, h].double() if carry else None
            go = s["grad_out"][b, :, h].double() if grads else None
            for r0 in range(0, T, R):
                r1 = min(T, r0 + R)
                c0 = max(0, int(begins[r0]))
                age = (torch.arange(r0, r1, device=DEV)[:, None] - torch.arange(c0, r1, device=DEV)[None, :]).double()
                w = torch.exp(-rate * age.clamp(min=0)) * ((age >= 0) & (ep[r0:r1, None] == ep[None, c0:r1]))
                w = w * scale
                a = (q[r0:r1] @ k[c0:r1].T) * w
                out[b, r0:r1, h] = a @ v[c0:r1]
                t = torch.arange(r0, r1, device=DEV).double() + 1
                w0 = torch.exp(-rate * t) * (ep[r0:r1] == -1) * scale
                if carry:
                    out[b, r0:r1, h] += w0[:, None] * (q[r0:r1] @ s0)
                if grads:
                    da = go[r0:r1] @ v[c0:r1].T
                    dlog[h] += (age * a * da).sum()
                    dvv[b, c0:r1, kh] += a.T @ go[r0:r1]
                    da = da * w
                    dq[b, r0:r1, h] += da @ k[c0:r1]
                    dkk[b, c0:r1, kh] += da.T @ q[r0:r1]
                    if carry:
                        dq[b, r0:r1, h] += w0[:, None] * (go[r0:r1] @ s0.T)
                        into = (q[r0:r1] * w0[:, None]).T @ go[r0:r1]
                        dstate[b, h] += into
                        dlog[h] += (((q[r0:r1] * (w0 * t)[:, None]).T @ go[r0:r1]) * s0).sum()
            # the state after the last step
            age = (T - 1 - torch.arange(T, device=DEV)).double()
            w = torch.exp(-rate * age) * (ep == ep[-1])
            state[b, h] = (k * w[:, None]).T @ v
            on = 1.0 if carry and begins[-1] == -1 else 0.0
            if on:
                state[b, h] += math.exp(-rate * T) * s0
            if grads and s["grad_state"] is not None:
                gs = s["grad_state"][b, h].double()
                dkk[b, :, kh] += w[:, None] * (v @ gs.T)
                dvv[b, :, kh] += w[:, None] * (k @ gs)
                dlog[h] += (((k * (w * age)[:, None]).T @ v) * gs).sum()
                if on:
                    dstate[b, h] += math.exp(-rate * T) * gs
                    dlog[h] += T * math.exp(-rate * T) * (s0 * gs).sum()
    if not grads:
        return {"out": out, "state": state}
    r = {"out": out, "dq": dq, "dk": dkk, "dv": dvv, "dalpha": -torch.sign(s["alpha"]).double() * dlog}
    return {**r, "dstate": dstate} if carry else r


def _exact_step(s):
    c = s["case"]
    G = c["H"] // c["Hk"]
    gamma = torch.exp(-s["alpha"].double().abs())
    out = torch.empty(c["B"], c["H"], c["dv"], dtype=torch.float64, device=DEV)
    state = torch.empty(s["state"].shape, dtype=torch.float64, device=DEV)
    for h in range(c["H"]):
        q, k, v = s["q"][:, h].double(), s["k"][:, h // G].double(), s["v"][:, h // G].double()
        before = torch.where((s["start"] != 0)[:, None, None], 0.0, gamma[h] * s["state"][:, h].double())
        state[:, h] = before + k[:, :, None] * v[:, None, :]
        # q (before + k^T v), without the sum over the new state
        out[:, h] = s["scale"] * ((q[:, :, None] * before).sum(1) + (q * k).sum(1, keepdim=True) * v)
    return {"out": out, "state": state}


def _exact_rotate(s, grads):
    """Pairs as complex numbers turned by exp(i position freq)."""
    c = s["case"]
    rot = c["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       s["positions"].double()[..., None, None] * s["freq"].double())

    def split(x):
        z = x[..., :rot]
        z = z.unflatten(-1, (rot // 2, 2)) if c["interleaved"] else z.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        return torch.view_as_complex(z.contiguous())

    def join(z, rest):
        z = torch.view_as_real(z)
        z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, rest], -1)

    got = {}
    for name, w, g in (("q", s["wq"], s.get("gq")), ("k", s["wk"], s.get("gk"))):
        x = s[name].double()
        r = torch.ones((), dtype=torch.float64, device=DEV)
        wd = torch.ones(c["d"], dtype=torch.float64, device=DEV)
        if w is not None:
            r, wd = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS), w.double()
        y = x * r * wd
        got[name] = join(split(y) * turn, y[..., rot:])
        if grads:
            g = g.double()
            gy = join(split(g) * turn.conj(), g[..., rot:])
            if w is None:
                got["d" + name] = gy
            else:
                got["dw" + name] = (gy * x * r).sum((0, 1, 2))
                gy = gy * wd
                got["d" + name] = r * gy - x * r ** 3 * (gy * x).mean(-1, keepdim=True)
    return got


def exact(case, seed):
    # pairs of rows within reach of each other, at most
    if case["kind"] in ("scan", "train"):
        reach = min(case["T"], 4 * case["mean"] + 1024)
        if case["B"] * case["H"] * case["T"] * reach > (8e10 if case["kind"] == "scan" else 4e10):
            return None
    s = prepare(case, seed)
    if case["kind"] == "step":
        return _exact_step(s)
    if case["kind"] in ("scan", "train"):
        return _exact_scan(s, case["kind"] == "train")
    return _exact_rotate(s, case["kind"] == "rotate_train")
