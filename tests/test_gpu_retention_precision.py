"""Retention on the GPU: what it keeps of its inputs' and its decays' precision,
against the 64-bit recurrence (retention_ref.py) or a closed form."""
import numpy as np
import pytest

from test_gpu_retention import F32_TOL, Case

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dk,dv", [(8, 8), (64, 64), (64, 128), (128, 64), (128, 128), (80, 40)])
@pytest.mark.parametrize("T", [50, 300])
@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 2)])
def test_bf16_results_round_once(dk, dv, T, H, Hk):
    """A bf16 result is the sum in floats, rounded: 2^-8 of the result itself at most,
    not of its terms.  The terms keep what two bf16 planes hold, 2^-17 for the pairs'
    products or the state a row reads and 2^-17 more where a row went into the state,
    beside fp32's bound: (2 2^-17 + F32_TOL) of the sum over absolute values, and the
    rounding's 2^-8 of that error."""
    c = Case("bf16", 2, T, H, Hk, dk, dv, "some", True, seed=dk + dv + T, rates=[0.5, 0.1])
    got = c.run()
    r, m = c.expected()
    worst = {}
    for name in ("out", "dq", "dk", "dv"):
        err = np.abs(got[name].double().cpu().numpy() - r[name])
        allowed = 2.0 ** -8 * np.abs(r[name]) + (2.0 ** -16 + F32_TOL) * (1 + 2.0 ** -8) * m[name]
        worst[name] = float((err / allowed).max())
    print("  " + " ".join("%s %.2f" % w for w in worst.items()), flush=True)
    assert max(worst.values()) <= 1.0, worst


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128)])
@pytest.mark.parametrize("T", [50, 700])
def test_same_bits_whatever_else_is_asked_for(dtype, dk, dv, T):
    """The state after the tape, or a carried state of zeros and its gradient, change
    no bit of the other results."""
    c = Case(dtype, 1, T, 2, 1, dk, dv, "some", False, seed=T)
    args, g = c.gpu_args(), c.gpu["grad_out"]
    out = mb.scan_retention(*args, scale=c.scale)
    zeros = torch.zeros(1, 2, dk, dv, device=out.device)
    assert torch.equal(out, mb.scan_retention(*args, scale=c.scale, final_state=True)[0])
    assert torch.equal(out, mb.scan_retention(*args, scale=c.scale, state=zeros))
    for alpha in (False, True):
        alone = mb.scan_retention_bwd(*args, g, scale=c.scale, need_grad_alpha=alpha)
        with_state = mb.scan_retention_bwd(*args, g, scale=c.scale, state=zeros, grad_state=zeros, need_grad_alpha=alpha)
        for name, x, y in zip(("dq", "dk", "dv", "dalpha"), alone, with_state):
            assert (x is None and y is None) or torch.equal(x, y), (name, alpha)
