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
