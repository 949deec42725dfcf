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


class LongCase(Case):
    """More chunks than the bound above counts: 3 roundings for each of them."""

    def tol(self, name):
        chunks = (self.cpu["q"].shape[1] + 31) // 32
        f32 = (24 + 6 + 3 * chunks + 8) * 2.0 ** -24 + 2 * 2.0 ** -21
        return f32 if self.dtype == "f32" or name in ("state", "dalpha", "dstate") else 3 * 2.0 ** -8 + f32


@pytest.mark.parametrize("dtype,T", [("f32", 2100), ("f32", 4200), ("bf16", 4200), ("bf16", 8400)])
@pytest.mark.parametrize("begins", ["none", "some"])
def test_many_segments(dtype, T, begins):
    """More segments than the state scan's groups take at once, and than two turns
    of them: 66 and 132 of a chunk each."""
    assert segments(1, T, 2, dtype) - 1 in (66, 132)        # (the query counts the flags' bytes as one more)
    LongCase(dtype, 1, T, 2, 1, 32, 64, begins, True, seed=T, rates=[2e-4, 0.01]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 64), (128, 128), (72, 40)])
def test_segments_of_wide_heads(dtype, dk, dv):
    """Two classes of tiles in one gradient, shared heads, a state in and out."""
    LongCase(dtype, 1, 700, 4, 2, dk, dv, "some", True, seed=dk, rates=[1e-3, 0.05]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H", [(2, 40, 2), (1, 500, 2), (300, 70, 2)])
def test_single_segment_and_many_tapes(dtype, B, T, H):
    """One chunk, a few segments, one segment of several chunks (600 heads of
    tapes: enough workgroups without a second segment)."""
    LongCase(dtype, B, T, H, 1, 32, 40, "some", True, seed=B, rates=[0.02]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [30, 700])
@pytest.mark.parametrize("dk,dv", [(32, 64), (128, 128)])
@pytest.mark.parametrize("carry", [False, True])
def test_gradient_without_rates(dtype, T, dk, dv, carry):
    """need_grad_alpha=False is a pass of its own."""
    c = LongCase(dtype, 1, T, 2, 1, dk, dv, "some", carry, seed=T)
    g = c.gpu
    got = mb.scan_retention_bwd(*c.gpu_args(), g["grad_out"], scale=c.scale, state=g["state"], grad_state=g["grad_state"],
                                need_grad_alpha=False)
    assert got[3] is None
    r, m = c.expected()
    for name, y in zip(("dq", "dk", "dv", None, "dstate"), got):
        if y is not None:
            assert cond_err(y.double().cpu().numpy(), r[name], m[name]) <= c.tol(name), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 64), (128, 128)])
@pytest.mark.parametrize("what", ["q", "k", "v", "grad_out"])
@pytest.mark.parametrize("alpha", [False, True])
@pytest.mark.parametrize("begins", [False, True])
def test_nonfinite_values_in_later_segments(dtype, dk, dv, what, alpha, begins):
    """As above over several segments, the value in the third chunk or later, with
    and without the rates' gradient.  (dalpha is a sum over everything.)"""
    T = 400
    c = LongCase(dtype, 1, T, 2, 1, dk, dv, "none", True, seed=9)
    f = c.cpu["start"]
    if begins:
        f[:, [0, 20, 130, 170, 200, 300]] = 1
        c.gpu["start"] = torch.from_numpy(f).to(DEV)
    x = c.gpu[what].clone()
    x[0, 180, 0, 7] = float("nan")
    x[0, 199, 0, 3] = float("inf")
    c.put(what, x.cpu())
    g = c.gpu
    out, S = mb.scan_retention(*c.gpu_args(), scale=c.scale, state=g["state"], final_state=True)
    dq, dk_, dv_, da, ds = mb.scan_retention_bwd(*c.gpu_args(), g["grad_out"], scale=c.scale, state=g["state"],
                                                 grad_state=g["grad_state"], need_grad_alpha=alpha)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        r, _ = c.expected()
    x = c.cpu[what]
    x[~np.isfinite(x)] = 1.0
    m = ref.magnitudes(*c.ref_args(), c.cpu["grad_out"], c.cpu["state"], c.cpu["grad_state"])
    for name, y in (("out", out), ("state", S), ("dq", dq), ("dk", dk_), ("dv", dv_), ("dalpha", da), ("dstate", ds)):
        if y is None:
            continue
        y = y.double().cpu().numpy()
        fine = np.isfinite(r[name])
        assert np.array_equal(np.isfinite(y), fine), name
        assert cond_err(y[fine], r[name][fine], m[name][fine]) <= c.tol(name), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("same_episode", [True, False])
def test_products_that_the_mask_leaves_out_may_overflow(dtype, same_episode):
    """A query of 1e20 before a key of 1e20: their product is no part of anything,
    and is infinite."""
    c = Case(dtype, 1, 100, 2, 2, 32, 32, "none", True, seed=13)
    if not same_episode:
        c.cpu["start"][0, 41] = 1
        c.gpu["start"] = torch.from_numpy(c.cpu["start"]).to(DEV)
    q, k = c.gpu["q"].clone(), c.gpu["k"].clone()
    q[0, 37, :, 5] = 1e20
    k[0, 37, :, 5] = 0.5
    k[0, 45, :, 5] = 1e20
    q[0, 45, :, 5] = 0.5
    c.put("q", q.cpu())
    c.put("k", k.cpu())
    c.check()


def test_dalpha_to_its_own_size():
    """dalpha's bound above is its terms' sizes, which mostly cancel.  Against the
    gradient itself: a head's terms add up like a walk of n steps, so that errors of
    half a step of float each, independent, leave about 2^-24 of it, and a row of
    sums of 8 roundings one after the other 8 2^-24; with the planes' 2^-21 of a pair
    of floats, 2^-20 = 1e-6 of the largest |dalpha|.  Five times that."""
    for dtype in ("f32", "bf16"):
        c = LongCase(dtype, 2, 600, 4, 2, 64, 64, "some", True, seed=17, rates=[1e-3, 0.01, 0.05, 0.3])
        da = c.run()["dalpha"].double().cpu().numpy()
        r, _ = c.expected()
        e = np.abs(da - r["dalpha"]).max() / np.abs(r["dalpha"]).max()
        print("  dalpha %.1e" % e, flush=True)
        assert e <= 5e-6


def test_two_threads_on_two_streams():
    """Calls at once, each on its own stream: the bits of the calls alone."""
    import threading
    cases = [Case("bf16", 2, 500, 4, 2, 64, 64, "some", True, seed=40),
             Case("f32", 1, 900, 2, 2, 32, 64, "some", True, seed=41)]
    alone = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(5):
                    got[i] = cases[i].run()
        except Exception as e:      # noqa: BLE001 -- handed to the test below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for a, b in zip(alone, got):
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_two_graphs_of_training_steps():
    """Forward and backward through autograd captured twice, with inputs of their
    own, replayed in turn with eager calls between: the eager results each time."""
    cases = [Case("bf16", 1, 300, 4, 2, 64, 64, "some", False, seed=50 + i) for i in range(2)]

    def step(c):
        x = [c.gpu[n].detach().requires_grad_(True) for n in ("q", "k", "v", "alpha")]
        out = mb.retention(*x, c.gpu["start"], scale=c.scale)
        return (out,) + torch.autograd.grad(out, x, c.gpu["grad_out"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c in cases:
            step(c)
    torch.cuda.current_stream().wait_stream(s)
    graphs, results = [], []
    for c in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            results.append([y.detach() for y in step(c)])
    for i in range(4):
        for c in cases:
            for n in ("q", "v", "grad_out"):
                c.gpu[n].copy_(torch.roll(c.gpu[n], 1 + i, 1))
        for j in (0, 1) if i % 2 else (1, 0):
            graphs[j].replay()
        torch.cuda.synchronize()
        for c, y in zip(cases, results):
            for a, b in zip(step(c), y):
                assert torch.equal(a, b)


def test_more_than_2_31_elements():
    """A tape whose last rows lie past 2^31 elements and 2^32 bytes: the rows behind
    its last begin against the formula, all of them finite."""
    T, H, d, tail = 560000, 32, 128, 70
    announce("retention T=%d H=%d d=%d bf16" % (T, H, d))
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = [torch.empty(1, T, H, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(4)]
    assert x[0].numel() > 1 << 31
    alpha = torch.linspace(0.001, 0.1, H, device=DEV)
    start = torch.zeros(1, T, dtype=torch.uint8, device=DEV)
    start[0, T - tail] = 1
    out, S = mb.scan_retention(*x[:3], alpha, start, final_state=True)
    got = mb.scan_retention_bwd(*x[:3], alpha, start, x[3])
    for y in (out, S) + got[:4]:
        assert bool(torch.isfinite(y.sum(dtype=torch.float32)))
    heads = [0, H - 1]
    cut = [t[:, T - tail:, heads].double().cpu().numpy() for t in x]
    args = (*cut[:3], alpha[heads].double().cpu().numpy(), start[:, T - tail:].cpu().numpy(), d ** -0.5)
    r = ref.forward(*args)
    b = ref.backward(*args, cut[3])
    m = ref.magnitudes(*args, cut[3])
    for name, y, want in (("out", out, r[0]), ("dq", got[0], b["dq"]), ("dk", got[1], b["dk"]), ("dv", got[2], b["dv"])):
        y = y[:, T - tail:, heads].double().cpu().numpy()
        assert cond_err(y, want, m[name]) <= BF16_TOL, name
    assert cond_err(S[:, heads].double().cpu().numpy(), r[1], m["state"]) <= F32_TOL


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_of_a_large_batch(dtype):
    """More rows than a grid has in y or z; rows that begin among them."""
    B, H, d = 70001, 2, 32
    announce("retention step B=%d" % B)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    q, k, v = (torch.randn(B, H, d, generator=g, device=DEV).to(DT[dtype]) for _ in range(3))
    S = torch.randn(B, H, d, d, generator=g, device=DEV)
    start = (torch.rand(B, generator=g, device=DEV) < 0.3).to(torch.uint8)
    alpha = torch.tensor([0.1, -0.5], device=DEV)
    keep = torch.where(start[:, None].bool(), 0.0, torch.exp(-alpha.double().abs())[None])
    old = keep[:, :, None, None] * S.double()
    want = old + k.double()[..., None] * v.double()[:, :, None]
    m = old.abs() + (k.double()[..., None] * v.double()[:, :, None]).abs()
    out = mb.retention_step(q, k, v, alpha, S, start)
    assert float(((S.double() - want).abs() / torch.maximum(want.abs(), m)).max()) <= 3 * 2.0 ** -24 * 1.01
    o = (q.double()[..., None] * want).sum(2) * d ** -0.5
    mo = (q.double().abs()[..., None] * m).sum(2) * d ** -0.5
    e = float(((out.double() - o).abs() / mo).max())
    assert e <= F32_TOL + (0 if dtype == "f32" else 2.0 ** -8), e


def test_step_marks_the_state_as_changed():
    """A graph that saved the state before the step must not use it after."""
    c = Case("f32", 1, 20, 2, 2, 32, 32, "none", True, seed=2)
    g = c.gpu
    v = g["v"].clone().requires_grad_(True)
    S = g["state"].clone()
    out = mb.retention(g["q"], g["k"], v, g["alpha"], g["start"], state=S)
    mb.retention_step(*(g[n][:, 0].contiguous() for n in "qkv"), g["alpha"], S)
    with pytest.raises(RuntimeError):
        out.sum().backward()


def test_second_derivative_is_refused():
    c = Case("f32", 1, 20, 2, 2, 32, 32, "none", False, seed=2)
    g = c.gpu
    v = g["v"].clone().requires_grad_(True)
    out = mb.retention(g["q"], g["k"], v, g["alpha"], g["start"])
    dv, = torch.autograd.grad(out.square().sum(), v, create_graph=True)
    with pytest.raises(RuntimeError):
        dv.sum().backward()


def test_workspace_elsewhere_is_refused():
    c = Case("f32", 1, 20, 2, 2, 32, 32, "none", False, seed=2)
    with pytest.raises(ValueError):
        mb.scan_retention(*c.gpu_args(), workspace=torch.empty(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError):
        mb.scan_retention_bwd(*c.gpu_args(), c.gpu["grad_out"], workspace=torch.empty(1 << 24, dtype=torch.uint8))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0, 1, 70])
def test_gradient_without_query_heads(dtype, T):
    """Key heads that no query head reads have a gradient of zeros.  (The memory that
    the gradients get held other values before.)"""
    announce("retention bwd H=0 %s T=%d" % (dtype, T))
    k, v = (torch.randn(2, T, 3, d, device=DEV).to(DT[dtype]) for d in (64, 32))
    q, g = (torch.empty(2, T, 0, d, dtype=DT[dtype], device=DEV) for d in (64, 32))
    alpha, start = torch.empty(0, device=DEV), torch.zeros(2, T, dtype=torch.uint8, device=DEV)
    old = [torch.full_like(x, 7.0) for x in (k, v)]
    del old
    dq, dk, dv, da, ds = mb.scan_retention_bwd(q, k, v, alpha, start, g)
    assert dq.shape == q.shape and da.shape == (0,) and ds is None
    assert dk.shape == k.shape and dv.shape == v.shape and not bool(dk.any()) and not bool(dv.any())
    leaves = [x.clone().requires_grad_(True) for x in (q, k, v)]
    mb.retention(*leaves, alpha, start).backward(g)
    assert not bool(leaves[1].grad.any()) and not bool(leaves[2].grad.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hk", [1, 65535])
def test_most_heads_of_a_tape(dtype, Hk):
    """H = 65535 of 128 columns: a chunk's rows span just under 2^31 bytes where the
    gradients of shared heads are floats.  The first and last query heads' results, and
    the key heads' gradients as sums over all of them."""
    T, H, d = 65, 65535, 128
    announce("retention %s T=%d H=%d/%d d=%d" % (dtype, T, H, Hk, d))
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    q, k, v, go = (torch.randn(1, T, h, d, generator=g, device=DEV).to(DT[dtype]) for h in (H, Hk, Hk, H))
    alpha = torch.linspace(0.01, 0.3, H, device=DEV)
    start = torch.zeros(1, T, dtype=torch.uint8, device=DEV)
    start[0, [0, 20, 64]] = 1
    out = mb.scan_retention(q, k, v, alpha, start)
    dq, dk, dv, da, _ = mb.scan_retention_bwd(q, k, v, alpha, start, go)
    heads = [0, 1, H - 1]
    cut = [t[:, :, heads if t.shape[2] == H else [0, 0, 0]].double().cpu().numpy() for t in (q, k, v, go)]
    args = (*cut[:3], alpha[heads].double().cpu().numpy(), start.cpu().numpy(), d ** -0.5)
    r, b, m = ref.forward(*args)[0], ref.backward(*args, cut[3]), ref.magnitudes(*args, cut[3])
    tol = F32_TOL if dtype == "f32" else BF16_TOL
    for name, y, want in (("out", out, r), ("dq", dq, b["dq"])) + ((("dk", dk, b["dk"]), ("dv", dv, b["dv"])) if Hk == H else ()):
        assert cond_err(y[:, :, heads].double().cpu().numpy(), want, m[name]) <= tol, name
    assert cond_err(da[heads].double().cpu().numpy(), b["dalpha"], m["dalpha"]) <= F32_TOL
    if Hk == 1:                                            # the last step alone: dk = scale v (q . q's head's gradient)
        p = (go[0, 64].double() @ v[0, 64, 0].double()) * d ** -0.5
        want = (p[:, None] * q[0, 64].double()).sum(0)
        size = (p.abs()[:, None] * q[0, 64].double().abs()).sum(0)
        e = float(((dk[0, 64, 0].double() - want).abs() / torch.maximum(size, want.abs())).max())
        # a sum of 65535 floats, one after the other: as a walk of as many roundings
        assert e <= tol + 5 * 2.0 ** -24 * 65535 ** 0.5, e


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_tapes(dtype):
    """B = 32767: the largest grid of a launch for both directions at once."""
    LongCase(dtype, 32767, 3, 2, 1, 8, 16, "some", True, seed=12).check()
