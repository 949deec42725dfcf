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
