"""The gated recurrence where decays, gates and values come near the ends of their types, on
the GPU against gated_ref.py, with the tolerances of test_gpu_gated.py (E = 2^-24).  Where
gates are larger than 8, in bf16, a sigmoid is off by another |v| E of itself (its
exponential's argument is one rounded product)."""
import numpy as np
import pytest

import gated_ref as ref
from conftest import announce, cond_err
from test_gpu_gated import DEV, DT, E, inputs, np64, tol

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu


def run(s):
    c = {k: None if v is None else v.to(DEV) for k, v in s.items()}
    h, last, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], final_state=True, keep_states=True)
    got = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    torch.cuda.synchronize()
    return h, last, kept, dict(zip(("x", "gates", "alpha", "state"), got))


def expected(s):
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    h = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    return h, ref.grads(a["x"], a["gates"], a["alpha"], a["start"], a["grad_h"], a["state"], a["grad_state"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("alpha,r", [(1e-30, 0.0), (1e-33, 0.0), (1e-35, 0.0), (1.0, -75.0), (1e-3, -75.0), (0.3, -60.0)])
def test_next_to_no_decay(dtype, alpha, r):
    """Inputs are weighed by m, about sqrt(2 u), whatever u is: states that start at zero and
    the gradients of x and the gates are right relative to themselves."""
    announce("gated next to no decay %s alpha=%g r=%g" % (dtype, alpha, r))
    T = 300
    s = inputs(dtype, 2, T, 68, "some", False, 7, rates=(alpha, alpha))
    s["gates"][:, :, 0] += r
    h, last, kept, got = run(s)
    (rh, mh, rl, ml), want = expected(s)
    more = 0.0 if dtype == "f32" else -(r - 8) * E
    assert cond_err(np64(h), rh, mh) <= tol(dtype, T) + more
    assert cond_err(np64(last), rl, ml) <= tol(dtype, T, rounded=False) + more
    for name, y in got.items():
        assert cond_err(np64(y), *want[name]) <= tol(dtype, T, True, name in ("x", "gates")) + 2 * more, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_inputs_where_nothing_decays(dtype):
    """No rate or a gate of -inf lets nothing in: no gradient of x and the gates, whatever x
    and the gradient that arrives are, and the state's goes through."""
    announce("gated large inputs without a decay %s" % dtype)
    T, d = 200, 8
    s = inputs(dtype, 1, T, d, "none", True, 2)
    s["x"] = torch.full((1, T, d), 2.0 ** 70, dtype=DT[dtype])
    s["grad_h"] = torch.full((1, T, d), 2.0 ** 60, dtype=DT[dtype])
    s["alpha"][:4] = 0.0
    s["gates"][:, :, 0, 4:] = -float("inf")
    h, last, _, got = run(s)
    assert torch.equal(last.cpu(), s["state"]) and bool((h == last[:, None].to(h.dtype)).all())
    for name in ("x", "gates", "alpha"):
        assert not bool(got[name].any()), name
    total = np64(s["grad_state"]) + T * 2.0 ** 60
    assert np.abs(np64(got["state"]) / total - 1).max() <= T * E


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rates", [(1.0, 1e-3), (50.0, 0.6)])
def test_large_gates(dtype, rates):
    """Finite gates up to 40 either way.  In bf16 a sigmoid is off by another 40 E, b by that of
    both its gates, half of the first's through m (60 E), and what a decay takes by 40 E: 100 E
    in a state, twice that in gradients.  Decays down to exp(-50) and sigmoids of -40 take
    products of gradients below the normal range (some are 1e-48): each is off by 2^-149 there,
    which factors up to 50 and sums over 400 steps make 2^-134 at most, E of 2^-110: magnitudes
    count as that at least."""
    announce("gated large gates %s rates=%s" % (dtype, rates))
    T = 400
    s = inputs(dtype, 2, T, 64, "some", True, 9, rates=rates)
    s["gates"] = (s["gates"].float() * 20.0).clamp(-40.0, 40.0).to(DT[dtype])
    more = 0.0 if dtype == "f32" else 100 * E
    h, last, kept, got = run(s)
    (rh, mh, rl, ml), want = expected(s)
    assert cond_err(np64(h), rh, mh) <= tol(dtype, T) + more
    assert cond_err(np64(last), rl, ml) <= tol(dtype, T, rounded=False) + more
    for name, y in got.items():
        r, m = want[name]
        assert cond_err(np64(y), r, np.maximum(m, 2.0 ** -110)) <= tol(dtype, T, True, name in ("x", "gates")) + 2 * more, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("u", [0.4, 0.6, 3.0, 20.0])
def test_what_decays_leave(dtype, u):
    """A state that nothing is added to, by itself: each step's decay leaves a, off by u E
    where it is fast, what it takes by 11 E where it is slow, and rounds twice."""
    announce("gated what is left %s u=%g" % (dtype, u))
    steps, d = 4, 64
    alpha = torch.full((d,), 2 * u, device=DEV)
    gates = torch.zeros(1, steps, 2, d, device=DEV, dtype=DT[dtype])
    gates[:, :, 1] = -float("inf")
    x, start = torch.ones(1, steps, d, device=DEV, dtype=DT[dtype]), torch.zeros(1, steps, dtype=torch.uint8, device=DEV)
    state = torch.rand(1, d, device=DEV) + 0.5
    _, last = mb.scan_gated(x, gates, alpha, start, state, final_state=True)
    row = state.clone()
    for t in range(steps):
        mb.gated_step(x[:, t].contiguous(), gates[:, t].contiguous(), alpha, row)
    want = np64(state) * np.exp(-steps * 0.5 * np64(alpha))
    # (sigmoid(0) is right to 6 E, so u is: 7 E of it; the run's decay goes by the sum of its rates)
    bound = (steps * (8 * u + 11 + 2) + 16) * E
    for got in (last, row):
        assert np.abs(np64(got) / want - 1).max() <= bound


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rates", [(0.4, 1e-3), (50.0, 0.6)])
def test_bad_states_stay_in_their_episode(bad, dtype, rates):
    """A state that is not finite stays so in its feature until the next begin step, forwards
    and in the gradients; at a begin step nobody looks at it."""
    announce("gated state %s %s rates=%s" % (bad, dtype, rates))
    T, d = 500, 20
    s = inputs(dtype, 2, T, d, "none", True, 1, rates=rates)
    s["gates"][:] = s["gates"].clamp(-1, 1)
    s["gates"][:, :, 0] = -4.0                                       # (so that nothing decays to nothing)
    s["start"][:, 300] = 1
    s["start"][1, 0] = 1
    s["state"][:, 7] = bad
    h, last, kept, got = run(s)
    ok = torch.isfinite(h.float())
    if rates[0] < 0.5:
        assert not bool(ok[0, :300, 7].any())
    ok[0, :300, 7] = True
    assert bool(ok.all()) and bool(torch.isfinite(last).all())
    for name, t in (("x", got["x"]), ("gates", got["gates"])):
        ok = torch.isfinite(t.float())
        ok[0, :300, ..., 7] = True
        assert bool(ok.all()), name
    assert bool(torch.isfinite(got["state"]).all())
    ok = torch.isfinite(got["alpha"])
    ok[7] = True
    assert bool(ok.all())
    row = s["state"].to(DEV)
    y = mb.gated_step(s["x"][:, 0].contiguous().to(DEV), s["gates"][:, 0].contiguous().to(DEV), s["alpha"].to(DEV), row,
                      torch.tensor([0, 1], dtype=torch.uint8, device=DEV))
    ok = torch.isfinite(y.float())
    assert not bool(ok[0, 7])
    ok[0, 7] = True
    assert bool(ok.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,d", [(2, 131, 70), (3, 31, 2), (1, 60, 130), (2, 200, 256), (2, 64, 66)])
def test_nothing_behind_even_rows(dtype, B, T, d):
    """Rows of pairs at even addresses, whose last columns fill a chain partly or wholly:
    guards around every output, and behind the workspaces."""
    announce("gated guards of even rows %s B=%d T=%d d=%d" % (dtype, B, T, d))
    s = inputs(dtype, B, T, d, "some", True, 6)
    want = mb.scan_gated(*(s[k].to(DEV) for k in ("x", "gates", "alpha", "start", "state")), final_state=True, keep_states=True)
    want += mb.scan_gated_bwd(*(s[k].to(DEV) for k in ("x", "gates", "alpha", "start")), want[2], s["grad_h"].to(DEV),
                              s["grad_state"].to(DEV))

    def shifted(t):
        buf = torch.full((t.numel() + 132,), 7, dtype=t.dtype, device=DEV)
        view = buf[66:66 + t.numel()].view(t.shape)
        view.copy_(t)
        return buf, view

    p = {k: shifted(v)[1] for k, v in s.items()}
    outs = [shifted(torch.zeros_like(t)) for t in want]
    o = [v.data_ptr() for _, v in outs]
    dt = mb.F32 if dtype == "f32" else mb.BF16
    n = max(mb.memoroid_scan_gated_workspace_bytes(B, T, d, dt), mb.memoroid_scan_gated_bwd_workspace_bytes(B, T, d, dt))
    ws = torch.randint(0, 256, (n + 512,), dtype=torch.uint8, device=DEV)
    keep = ws[n:].clone()
    st = torch.cuda.current_stream().cuda_stream
    a = [p[k].data_ptr() for k in ("x", "gates", "alpha", "start", "state", "grad_h", "grad_state")]
    assert mb.memoroid_scan_gated(*a[:5], o[0], o[1], o[2], B, T, d, dt, ws.data_ptr(), n, st) == mb.OK
    assert mb.workspace_status(ws) == mb.OK
    assert mb.memoroid_scan_gated_bwd(*a[:4], o[2], a[5], a[6], o[3], o[4], o[5], o[6], B, T, d, dt, ws.data_ptr(), n,
                                      st) == mb.OK
    assert mb.workspace_status(ws) == mb.OK
    for (buf, view), w in zip(outs, want):
        assert torch.equal(view, w)
        assert bool((buf[:66] == 7).all()) and bool((buf[66 + w.numel():] == 7).all())
    assert torch.equal(ws[n:], keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("B,d", [(3, 70), (2, 256), (5, 33), (1, 1)])
def test_step_at_any_address(dtype, shift, B, d):
    """A step's operands at any element, guards around what it writes."""
    announce("gated step guards %s shift=%d B=%d d=%d" % (dtype, shift, B, d))
    s = inputs(dtype, B, 1, d, "dense", True, 3)
    t = dict(x=s["x"][:, 0], gates=s["gates"][:, 0], alpha=s["alpha"], state=s["state"], start=s["start"][:, 0])
    c = {k: v.contiguous().to(DEV) for k, v in t.items()}
    state = c["state"].clone()
    want = mb.gated_step(c["x"], c["gates"], c["alpha"], state, c["start"])
    at = {}
    for k, v in (*c.items(), ("h", torch.zeros_like(want))):
        buf = torch.full((v.numel() + 64 + shift,), 7, dtype=v.dtype, device=DEV)
        buf[32 + shift:32 + shift + v.numel()] = v.flatten()
        at[k] = buf
    p = {k: v.data_ptr() + (32 + shift) * v.element_size() for k, v in at.items()}
    assert mb.memoroid_gated_step(p["x"], p["gates"], p["alpha"], p["start"], p["state"], p["h"], B, d,
                                  mb.F32 if dtype == "f32" else mb.BF16, torch.cuda.current_stream().cuda_stream) == mb.OK
    for k, w in (("h", want), ("state", state)):
        buf = at[k]
        assert torch.equal(buf[32 + shift:32 + shift + w.numel()].view(w.shape), w)
        assert bool((buf[:32 + shift] == 7).all()) and bool((buf[32 + shift + w.numel():] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_runs_of_many_chains_are_equal(dtype):
    """As many chains as one wavefront looks back for alone, and other work between the runs."""
    announce("gated equal runs of many chains %s" % dtype)
    s = inputs(dtype, 1, 16384, 1100, "none", True, 9)
    c = {k: v.to(DEV) for k, v in s.items()}
    first = None
    for turn in range(8):
        got = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], final_state=True, keep_states=True)
        got += mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], got[2], c["grad_h"], c["grad_state"])
        if first is None:
            first = [t.clone() for t in got]
        assert all(torch.equal(x, y) for x, y in zip(first, got)), turn
        if turn % 2:
            c["x"].float().exp().sum()


def test_gradients_past_32_bits():
    """More than 2^31 values: alpha's and the state's gradient are those of the last tape
    alone.  A gradient that arrives in one tile of that tape alone, behind a begin step, leaves
    one row of sums that is not zero, so alpha's is the same bit for bit."""
    announce("gated gradients past 2^31 values")
    B, T, d = 9, 65536, 4096
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    bx, bg = torch.zeros(B, T, d, device=DEV, dtype=torch.bfloat16), torch.zeros(B, T, 2, d, device=DEV, dtype=torch.bfloat16)
    bs, alpha = torch.zeros(B, T, device=DEV, dtype=torch.uint8), torch.rand(d, device=DEV, generator=g) * 0.1
    bx[-1] = torch.randn(T, d, device=DEV, generator=g)
    bg[-1] = torch.randn(T, 2, d, device=DEV, generator=g)
    bs[-1, 1:] = (torch.rand(T - 1, device=DEV, generator=g) < 0.0001).to(torch.uint8)
    up, state = torch.zeros(B, d, device=DEV), torch.zeros(B, d, device=DEV)
    up[-1], state[-1] = torch.randn(d, device=DEV, generator=g), torch.randn(d, device=DEV, generator=g)
    lone = [t[-1:].contiguous() for t in (bx, bg, bs, state, up)]
    _, kept = mb.scan_gated(bx, bg, alpha, bs, state, keep_states=True)
    _, lkept = mb.scan_gated(lone[0], lone[1], alpha, lone[2], lone[3], keep_states=True)
    assert torch.equal(kept[-1], lkept[0])
    got = mb.scan_gated_bwd(bx, bg, alpha, bs, kept, bx, up)
    want = mb.scan_gated_bwd(lone[0], lone[1], alpha, lone[2], lkept, lone[0], lone[4])
    assert torch.equal(got[3][-1], want[3][0]) and bool(want[3].any()) and not bool(got[3][:-1].any())
    del got
    bs[-1, T - 64] = 1
    gh = torch.zeros_like(bx)
    gh[-1, T - 64:] = bx[-1, T - 64:]
    lone[2] = bs[-1:].contiguous()
    _, kept = mb.scan_gated(bx, bg, alpha, bs, state, keep_states=True)
    _, lkept = mb.scan_gated(lone[0], lone[1], alpha, lone[2], lone[3], keep_states=True)
    got = mb.scan_gated_bwd(bx, bg, alpha, bs, kept, gh, up)[2]
    want = mb.scan_gated_bwd(lone[0], lone[1], alpha, lone[2], lkept, gh[-1:].contiguous(), lone[4])[2]
    assert torch.equal(got, want) and bool(want.all())
