"""Retention on the GPU: what it keeps of its inputs' and its decays' precision,
against the 64-bit recurrence (retention_ref.py) or a closed form."""
import numpy as np
import pytest

from conftest import announce
from test_gpu_retention import DEV, F32_TOL, Case

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


def slow_rates(n):
    return torch.logspace(np.log10(1 / 3000), -5, n, dtype=torch.float64).float()


def decayed(rates, T):
    """gamma^t for t = 1 .. T, and the sum of gamma^0 .. gamma^(t - 1), [T, heads]."""
    r = rates.double()[None]
    t = torch.arange(1, T + 1, dtype=torch.float64)[:, None]
    return torch.exp(-r * t), torch.expm1(-r * t) / torch.expm1(-r)


def walk_bound(rates, T, per_step, more):
    """T steps of `per_step` roundings of at most 2^-24 each, as likely up as down: a
    variance of 2^-48 / 3 a rounding, which decays by gamma^2 a step where the steps
    add to the value; five standard deviations, and `more` single roundings."""
    n = torch.clamp(0.5 / rates.double(), max=float(T))
    return 5 * 2.0 ** -24 * torch.sqrt(per_step * n / 3) + more * 2.0 ** -24


def test_rows_with_bad_values_keep_slow_decays():
    """Every chunk holds a NaN, in a column of its own: all are walked row by row.  The
    other columns against the closed form, q = k = v = 1: 8 scale times the sum of
    gamma^n.  A row rounds twice (its decay, what it adds); the sum of 8
    products and the decay's own 2^-24: 12."""
    T, H = 16384, 512
    announce("retention row by row, T=%d H=%d" % (T, H))
    rates = slow_rates(H)
    one = torch.ones(1, T, H, 8, device=DEV)
    v = one.clone()
    v[0, 5::32, :, 7] = float("nan")
    out, S = mb.scan_retention(one, one, v, rates.to(DEV), torch.zeros(1, T, dtype=torch.uint8, device=DEV), scale=1.0,
                               final_state=True)
    want = decayed(rates, T)[1].to(DEV)
    bound = walk_bound(rates, T, 2, 12).to(DEV)
    e = (out[0, :, :, 3].double() / (8 * want) - 1).abs().amax(0) / bound
    print("  out %.2f" % float(e.max()), flush=True)
    assert float(e.max()) <= 1
    e = (S[0, :, 2, 3].double() / want[-1] - 1).abs() / bound
    assert float(e.max()) <= 1
    assert bool(torch.isnan(out[0, 5:, :, 7]).all())


def test_gradient_of_rows_with_bad_values_keeps_slow_decays():
    """k holds a NaN in every chunk, in one column: both halves of the tape go through
    the segments' states row by row, and the walk as well.  dq's other columns, with
    ones everywhere else, are those of the scan above."""
    T, H = 16384, 256
    announce("retention gradient row by row, T=%d H=%d" % (T, H))
    rates = slow_rates(H)
    one = torch.ones(1, T, H, 8, device=DEV)
    k = one.clone()
    k[0, 5::32, :, 7] = float("nan")
    dq = mb.scan_retention_bwd(one, k, one, rates.to(DEV), torch.zeros(1, T, dtype=torch.uint8, device=DEV), one, scale=1.0)[0]
    want = decayed(rates, T)[1].to(DEV)
    e = (dq[0, :, :, 3].double() / (8 * want) - 1).abs().amax(0) / walk_bound(rates, T, 2, 12).to(DEV)
    print("  dq %.2f" % float(e.max()), flush=True)
    assert float(e.max()) <= 1


@pytest.mark.parametrize("H,d", [(1, 8), (4, 128)])
def test_segment_states_keep_slow_decays(H, d):
    """A state of ones and nothing added to it: out_t is d gamma^t, through as many
    segments as there are, each of which rounds once as it takes the state on (both
    forms of the scan of segments); in its own segment a row rounds the state's decay,
    the sum of d equal products and the result: 8."""
    T = 32 * 512 // H
    announce("retention segments, T=%d H=%d d=%d" % (T, H, d))
    one, none = torch.ones(1, T, H, d, device=DEV), torch.zeros(1, T, H, d, device=DEV)
    start = torch.zeros(1, T, dtype=torch.uint8, device=DEV)
    worst = 0.0
    for rates in slow_rates(64).reshape(-1, H):
        out = mb.scan_retention(one, none, none, rates.to(DEV), start, scale=1.0, state=torch.ones(1, H, d, d, device=DEV))
        want = decayed(rates, T)[0].to(DEV)
        e = (out[0, :, :, 3].double() / (d * want) - 1).abs().max()
        worst = max(worst, float(e))
    bound = 2.0 ** -24 * (5 * (132 / 3) ** 0.5 + 8)        # 128 segments or groups of them, and 4 in a group
    print("  out %.1e of %.1e" % (worst, bound), flush=True)
    assert worst <= bound


def test_steps_keep_slow_decays():
    """16384 steps of q = k = v = 1 against the closed form, 8 scale times the sum of
    gamma^n, and against the scan of the same steps (whose own bound comes on top).
    Two roundings a step, the sum of 8 products and the decay's own 2^-24."""
    T, H = 16384, 64
    announce("retention %d steps" % T)
    rates = torch.cat([slow_rates(H - 3), torch.tensor([1 / 3000, 1 / 4096, 1 / 51200])])
    one, alpha = torch.ones(1, H, 8, device=DEV), rates.to(DEV)
    S = torch.zeros(1, H, 8, 8, device=DEV)
    for _ in range(T):
        out = mb.retention_step(one, one, one, alpha, S, scale=1.0)
    want, bound = decayed(rates, T)[1][-1], walk_bound(rates, T, 2, 12)
    e = (out[0, :, 3].double().cpu() / (8 * want) - 1).abs() / bound
    print("  out %.2f" % float(e.max()), flush=True)
    assert float(e.max()) <= 1
    many = torch.ones(1, T, H, 8, device=DEV)
    scan, last = mb.scan_retention(many, many, many, alpha, torch.zeros(1, T, dtype=torch.uint8, device=DEV), scale=1.0,
                                   final_state=True)
    for x, y in ((out, scan[:, -1]), (S, last)):
        e = (x.double() / y.double() - 1).abs().reshape(H, -1).amax(1).cpu()
        assert bool((e <= bound + F32_TOL).all())
