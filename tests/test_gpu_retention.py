"""Retention on the GPU against the 64-bit recurrence (retention_ref.py), error
relative to max(|r|, m) with m the same sums over absolute values.

Tolerances.  fp32: a value passes through a sum over the head (4 products of 32
columns in 6 instructions each), one over a chunk's 32 rows, at most 3 roundings
per chunk of the state's carry and the planes' dropped 2^-21: with up to 64
chunks of 32 rows below (24 + 6 + 192 + 8) 2^-24 + 2 * 2^-21 = 1.5e-5, so 2e-5.
bf16: the output's rounding, one of the pairs' weights and one of the state, each
2^-8 at most: 3 * 2^-8, and the fp32 part.  The states and dalpha are fp32
results in both."""
import numpy as np
import pytest

import retention_ref as ref
from conftest import announce, cond_err

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32_TOL = 2e-5
BF16_TOL = 3 * 2.0 ** -8 + F32_TOL
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def flags(kind, B, T, rng):
    f = np.zeros((B, T), np.uint8)
    if kind == "short":
        f[rng.random((B, T)) < 0.2] = 1
    elif kind == "some":
        f[rng.random((B, T)) < 0.01] = 255
    elif kind == "all":
        f[:] = 1
    elif kind == "edges":
        f[:, ::32] = 3
        f[:, 63::64] = 1
    elif kind == "last":
        f[:, -1] = 1
    elif kind != "none":
        raise ValueError(kind)
    return f


class Case:
    """Inputs on the CPU in 64 bits (as the dtype holds them) and on the GPU."""

    def __init__(self, dtype, B, T, H, Hk, dk, dv, begins="some", carry=True, seed=0, rates=None, scale=None):
        announce("retention %s B=%d T=%d H=%d/%d dk=%d dv=%d %s carry=%s" % (dtype, B, T, H, Hk, dk, dv, begins, carry))
        rng = np.random.default_rng(seed)
        self.dtype = dtype
        self.dt = DT[dtype]
        self.gpu, self.cpu = {}, {}
        for name, shape, dt in (("q", (B, T, H, dk), self.dt), ("k", (B, T, Hk, dk), self.dt), ("v", (B, T, Hk, dv), self.dt),
                                ("grad_out", (B, T, H, dv), self.dt), ("state", (B, H, dk, dv), torch.float32),
                                ("grad_state", (B, H, dk, dv), torch.float32)):
            if not carry and name.endswith("state"):
                self.gpu[name] = self.cpu[name] = None
                continue
            self.put(name, torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dt))
        a = np.exp(rng.uniform(np.log(1e-3), np.log(0.5), H)) if rates is None else np.resize(rates, H)
        a = (a * np.where(np.arange(H) % 2, -1, 1)).astype(np.float32)
        self.put("alpha", torch.from_numpy(a))
        self.cpu["start"] = flags(begins, B, T, rng)
        self.gpu["start"] = torch.from_numpy(self.cpu["start"]).to(DEV)
        self.scale = float(dk ** -0.5 if scale is None else scale)

    def put(self, name, t):
        self.gpu[name] = t.to(DEV)
        self.cpu[name] = t.double().numpy()

    def ref_args(self):
        c = self.cpu
        return c["q"], c["k"], c["v"], c["alpha"], c["start"], self.scale

    def gpu_args(self):
        g = self.gpu
        return g["q"], g["k"], g["v"], g["alpha"], g["start"]

    def tol(self, name):
        return F32_TOL if self.dtype == "f32" or name in ("state", "dalpha", "dstate") else BF16_TOL

    def expected(self):
        c = self.cpu
        out, S, _ = ref.forward(*self.ref_args(), c["state"])
        r = dict(out=out, state=S, **ref.backward(*self.ref_args(), c["grad_out"], c["state"], c["grad_state"]))
        m = ref.magnitudes(*self.ref_args(), c["grad_out"], c["state"], c["grad_state"])
        return r, m

    def run(self):
        g = self.gpu
        out, S = mb.scan_retention(*self.gpu_args(), scale=self.scale, state=g["state"], final_state=True)
        dq, dk, dv, da, ds = mb.scan_retention_bwd(*self.gpu_args(), g["grad_out"], scale=self.scale, state=g["state"],
                                                   grad_state=g["grad_state"])
        torch.cuda.synchronize()
        return dict(out=out, state=S, dq=dq, dk=dk, dv=dv, dalpha=da, dstate=ds)

    def check(self):
        got = self.run()
        r, m = self.expected()
        errs = {}
        for name, y in got.items():
            if y is None:
                continue
            assert y.dtype == (torch.float32 if name in ("state", "dalpha", "dstate") else self.dt), name
            # gamma = exp(-200) is 1e-87: what is below fp32's smallest normal number
            # may come out as zero, an absolute error of 2^-126
            floor = 2.0 ** -126 / self.tol(name)
            errs[name] = cond_err(y.double().cpu().numpy(), r[name], np.maximum(m[name], floor))
        print("  " + " ".join("%s %.1e" % e for e in errs.items()), flush=True)
        for name, e in errs.items():
            assert e <= self.tol(name), (name, e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 127, 200])
def test_lengths(dtype, T):
    Case(dtype, 2, T, 2, 2, 64, 64, seed=T).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(8, 8), (64, 128), (128, 64), (128, 128), (80, 96), (96, 24), (40, 120)])
def test_head_widths(dtype, dk, dv):
    Case(dtype, 1, 100, 2, 2, dk, dv, seed=dk + dv).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 3), (4, 1), (6, 2), (8, 4)])
def test_shared_heads(dtype, H, Hk):
    Case(dtype, 2, 90, H, Hk, 32, 48, seed=H + Hk).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("begins", ["none", "short", "some", "all", "edges", "last"])
@pytest.mark.parametrize("carry", [False, True])
def test_flags(dtype, begins, carry):
    Case(dtype, 3, 150, 2, 1, 64, 64, begins, carry, seed=11).check()


@pytest.mark.parametrize("dtype,T", [("f32", 32 * 4 + 1), ("f32", 1000), ("f32", 2048), ("bf16", 64 * 4 + 1), ("bf16", 2000)])
@pytest.mark.parametrize("begins", ["none", "some"])
@pytest.mark.parametrize("carry", [False, True])
def test_segments(dtype, T, begins, carry):
    """Few heads and a longer tape: several segments, the last one ragged."""
    assert 1 < segments(1, T, 2, dtype)
    Case(dtype, 1, T, 2, 2, 32, 64, begins, carry, seed=T).check()


def segments(B, T, H, dtype):
    one = mb.memoroid_scan_retention_workspace_bytes(B, T, H, 32, 64, mb.F32 if dtype == "f32" else mb.BF16)
    return 1 + (one - 256) // (B * H * 32 * 64 * 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rates", [0.0, 1e-7, 3.0, 200.0, float("inf")])
def test_rates(dtype, rates):
    """No decay at all, one that 32 bits would lose from step to step, one that
    leaves a step or two, gamma = 0."""
    Case(dtype, 1, 300, 2, 2, 32, 32, "none", True, seed=5, rates=[rates]).check()


def test_slow_rate_over_a_long_tape():
    """gamma^T = exp(-1): the carry compounds over 1600 chunks.  Against the sum in
    closed form: q = k = v = 1 gives dk scale sum of gamma^n.  Every step of the
    carry rounds once, at most 2^-24 each and not one after the other the same way
    in all: 1600 2^-24 = 9.5e-5 if they all did; rounding to nearest spreads them
    as a walk, 40 2^-24, and 1e-5 is four times that."""
    T, rate = 51200, np.float32(1.0 / 51200)
    announce("retention slow rate T=%d" % T)
    one = torch.ones(1, T, 1, 8, device=DEV)
    a = torch.tensor([float(rate)], device=DEV)
    out = mb.scan_retention(one, one, one, a, torch.zeros(1, T, dtype=torch.uint8, device=DEV), scale=1.0)
    want = 8.0 * -np.expm1(-float(rate) * np.arange(1, T + 1)) / -np.expm1(-float(rate))
    got = out[0, :, 0, 3].double().cpu().numpy()
    assert np.abs(got / want - 1).max() <= 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["q", "k", "v", "grad_out", "state", "grad_state"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_nonfinite_values_stay_in_their_episode(dtype, what, value):
    """Every element that the recurrence leaves finite is finite and right, every
    other one is not finite."""
    c = Case(dtype, 1, 200, 2, 1, 32, 64, "none", True, seed=3)
    f = c.cpu["start"]
    f[:, [20, 70, 90, 100, 140, 163]] = 1
    c.gpu["start"] = torch.from_numpy(f).to(DEV)
    x = c.gpu[what].clone()
    if what.endswith("state"):
        x[0, 1, 3, 5] = value
    else:
        x[0, 80, 0, 7] = value
        x[0, 100, 0, 9] = value
        x[0, 162, 0, 2] = value
    c.put(what, x.cpu())
    got = c.run()
    with np.errstate(invalid="ignore"):
        r, _ = c.expected()
    # magnitudes of the same inputs with zeros in the bad places, for the finite elements
    x = c.cpu[what]
    x[~np.isfinite(x)] = 1.0
    m = ref.magnitudes(*c.ref_args(), c.cpu["grad_out"], c.cpu["state"], c.cpu["grad_state"])
    for name, y in got.items():
        y = y.double().cpu().numpy()
        fine = np.isfinite(r[name])
        assert np.array_equal(np.isfinite(y), fine), name
        assert cond_err(y[fine], r[name][fine], m[name][fine]) <= c.tol(name), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,dk,dv", [(1, 1, 1, 8, 8), (3, 4, 2, 64, 64), (5, 2, 1, 128, 128), (2, 3, 3, 80, 40)])
def test_steps(dtype, B, H, Hk, dk, dv):
    """Steps one by one are the scan, state and all; rows that begin forget."""
    T = 7
    c = Case(dtype, B, T, H, Hk, dk, dv, "short", True, seed=B)
    S = c.gpu["state"].clone()
    outs = []
    for t in range(T):
        q, k, v = (c.gpu[n][:, t].contiguous() for n in "qkv")
        outs.append(mb.retention_step(q, k, v, c.gpu["alpha"], S, c.gpu["start"][:, t].contiguous(), scale=c.scale))
    r, m = c.expected()
    # q S is a sum of 128 in float, the state a chain of 7 steps: below fp32's bound;
    # bf16 rounds the output alone
    e = cond_err(torch.stack(outs, 1).double().cpu().numpy(), r["out"], m["out"])
    assert e <= (F32_TOL if dtype == "f32" else 2.0 ** -8 + F32_TOL), e
    assert cond_err(S.double().cpu().numpy(), r["state"], m["state"]) <= F32_TOL


def test_step_without_flags_and_nonfinite_state():
    c = Case("f32", 2, 1, 2, 2, 64, 64, "none", True, seed=1)
    q, k, v = (c.gpu[n][:, 0].contiguous() for n in "qkv")
    S, S1 = c.gpu["state"].clone(), c.gpu["state"].clone()
    a = mb.retention_step(q, k, v, c.gpu["alpha"], S)
    b = mb.retention_step(q, k, v, c.gpu["alpha"], S1, torch.zeros(2, dtype=torch.uint8, device=DEV))
    assert torch.equal(a, b) and torch.equal(S, S1)
    S1[0] = float("nan")
    out = mb.retention_step(q, k, v, c.gpu["alpha"], S1, torch.tensor([9, 0], dtype=torch.uint8, device=DEV))
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(S1).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_steps(dtype):
    """A prompt read at once, its state carried on step by step, is the whole tape
    read at once."""
    c = Case(dtype, 2, 150, 4, 2, 64, 64, "some", False, seed=8)
    g = c.gpu
    cut = 141
    out, S = mb.scan_retention(*(g[n][:, :cut].contiguous() for n in "qkv"), g["alpha"], g["start"][:, :cut].contiguous(),
                               final_state=True)
    outs = [out]
    for t in range(cut, 150):
        q, k, v = (g[n][:, t].contiguous() for n in "qkv")
        outs.append(mb.retention_step(q, k, v, g["alpha"], S, g["start"][:, t].contiguous())[:, None])
    r, m = c.expected()
    assert cond_err(torch.cat(outs, 1).double().cpu().numpy(), r["out"], m["out"]) <= c.tol("out")
    assert cond_err(S.double().cpu().numpy(), r["state"], m["state"]) <= F32_TOL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("carry", [False, True])
def test_autograd(dtype, carry):
    c = Case(dtype, 2, 130, 4, 2, 64, 32, "some", carry, seed=21)
    g = c.gpu
    leaves = [g[n].clone().requires_grad_(True) if g[n] is not None else None for n in ("q", "k", "v", "alpha", "state")]
    got = mb.retention(*leaves[:4], g["start"], state=leaves[4], final_state=carry)
    if carry:
        torch.autograd.backward(got, (g["grad_out"], g["grad_state"]))
    else:
        got.backward(g["grad_out"])
    r, m = c.expected()
    for name, x in zip(("dq", "dk", "dv", "dalpha", "dstate"), leaves):
        if x is not None:
            assert cond_err(x.grad.double().cpu().numpy(), r[name], m[name]) <= c.tol(name), name


def test_autograd_of_the_state_alone():
    c = Case("f32", 1, 40, 2, 2, 32, 32, "none", True, seed=22)
    g = c.gpu
    v = g["v"].clone().requires_grad_(True)
    _, S = mb.retention(g["q"], g["k"], v, g["alpha"], g["start"], state=g["state"], final_state=True)
    S.backward(g["grad_state"])
    c.cpu["grad_out"] = np.zeros_like(c.cpu["grad_out"])
    r, m = c.expected()
    assert cond_err(v.grad.double().cpu().numpy(), r["dv"], m["dv"]) <= F32_TOL


def test_gradient_against_differences():
    """L = sum g out + sum G S along a random direction of every input: central
    differences of the kernels' own forward pass against the gradient.  The fp32
    forward's error (F32_TOL of the magnitude companions of L, about 10 |L|) over
    the step 2h = 0.02 leaves some 1e-2 of the derivative; 3e-2."""
    c = Case("f32", 2, 70, 2, 1, 32, 32, "some", True, seed=31)
    g = c.gpu
    names = ("q", "k", "v", "alpha", "state")
    rng = torch.Generator(device=DEV)
    rng.manual_seed(1)
    d = {n: torch.randn(g[n].shape, generator=rng, device=DEV) * (0.05 if n == "alpha" else 1.0) for n in names}

    def loss(t):
        x = {n: g[n] + t * d[n] for n in names}
        out, S = mb.scan_retention(x["q"], x["k"], x["v"], x["alpha"], g["start"], state=x["state"], final_state=True)
        return float((out.double() * g["grad_out"].double()).sum() + (S.double() * g["grad_state"].double()).sum())

    h = 0.01
    numeric = (loss(h) - loss(-h)) / (2 * h)
    grads = mb.scan_retention_bwd(*c.gpu_args(), g["grad_out"], state=g["state"], grad_state=g["grad_state"])
    want = sum(float((grads[i].double() * d[n].double()).sum()) for i, n in enumerate(names))
    scale = sum(float((grads[i].double() * d[n].double()).abs().sum()) for i, n in enumerate(names)) ** 0.5
    assert abs(numeric - want) <= 3e-2 * max(abs(want), scale), (numeric, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_again(dtype):
    """No order of sums depends on timing: two calls, and one on a workspace full of
    rubbish, give the same bits."""
    c = Case(dtype, 1, 1000, 2, 1, 64, 64, "some", True, seed=4)
    a, b = c.run(), c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n
    code = mb.F32 if dtype == "f32" else mb.BF16
    n = max(mb.memoroid_scan_retention_workspace_bytes(1, 1000, 2, 64, 64, code),
            mb.memoroid_scan_retention_bwd_workspace_bytes(1, 1000, 2, 1, 64, 64, code, 1))
    assert n <= mb.memoroid_workspace_bytes(mb.OP_RETENTION_BWD, 1, 1000, 2, 64, 64, 0)
    ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device=DEV)
    g = c.gpu
    out, S = mb.scan_retention(*c.gpu_args(), scale=c.scale, state=g["state"], final_state=True, workspace=ws)
    assert torch.equal(out, a["out"]) and torch.equal(S, a["state"])
    assert mb.workspace_status(ws) == mb.OK
    ws.random_(0, 256)
    got = mb.scan_retention_bwd(*c.gpu_args(), g["grad_out"], scale=c.scale, state=g["state"], grad_state=g["grad_state"],
                                workspace=ws)
    for n, y in zip(("dq", "dk", "dv", "dalpha", "dstate"), got):
        assert torch.equal(y, a[n]), n
    assert mb.workspace_status(ws) == mb.OK


def test_other_stream_and_empty_tapes():
    c = Case("bf16", 2, 300, 2, 2, 64, 64, "some", True, seed=6)
    a = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = c.run()
    s.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n]), n
    g = c.gpu
    none = [g[n][:, :0].contiguous() for n in "qkv"]
    out, S = mb.scan_retention(*none, g["alpha"], g["start"][:, :0].contiguous(), state=g["state"], final_state=True)
    assert out.shape == (2, 0, 2, 64) and torch.equal(S, g["state"])
    got = mb.scan_retention_bwd(*none, g["alpha"], g["start"][:, :0].contiguous(), g["grad_out"][:, :0].contiguous(),
                                state=g["state"], grad_state=g["grad_state"])
    assert torch.equal(got[4], g["grad_state"]) and not bool(got[3].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph(dtype):
    """Captured once, replayed with other inputs in the same place, eager work in
    between: every replay is the eager result."""
    c = Case(dtype, 1, 700, 2, 1, 64, 64, "some", True, seed=7)
    g = c.gpu
    c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run_no_sync = lambda: (mb.scan_retention(*c.gpu_args(), scale=c.scale, state=g["state"], final_state=True),
                                 mb.scan_retention_bwd(*c.gpu_args(), g["grad_out"], scale=c.scale, state=g["state"],
                                                       grad_state=g["grad_state"]))
        c.run_no_sync()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (out, S), grads = c.run_no_sync()
    for i in range(3):
        for n in ("q", "k", "v", "grad_out"):
            g[n].copy_(torch.roll(g[n], i + 1, 1))
        graph.replay()
        torch.cuda.synchronize()
        want = c.run()
        for n, y in zip(("out", "state", "dq", "dk", "dv", "dalpha", "dstate"), (out, S) + grads):
            assert torch.equal(y, want[n]), (i, n)
