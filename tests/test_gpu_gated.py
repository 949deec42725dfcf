"""The gated recurrence on the GPU against gated_ref.py, errors relative to max(|r|, m).

Tolerances, in E = 2^-24 (half a step of fp32, relative).  Forward: a sigmoid is off by
6 E (exponential 2 + 1 in its argument, sum 1, reciprocal 2), so u by 7, w by 11
(polynomial 4), m by 9 (half of w's, the root 2, the product 1), b by 17; a state's own
roundings, two a step, add up at random over an episode of n steps, 4 sqrt(n) with room;
a decay off by 11 E of what it takes moves a state by 11 E of its magnitude.  In all
(32 + 4 sqrt n) E.  Gradients go through two such chains and a / m: (72 + 8 sqrt n) E.
With bf16 inputs the exponential is off by another 1.5 |v| E, |v| < 8 here: 12 E in
each sigmoid, so twice the above, and bf16 results are rounded once, 2^-8."""
import numpy as np
import pytest

import gated_ref as ref
from conftest import announce, cond_err

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E = 2.0 ** -24


def tol(dtype, n, grad=False, rounded=True):
    t = (72 + 8 * n ** 0.5) * E if grad else (32 + 4 * n ** 0.5) * E
    return t if dtype == "f32" else 2 * t + (2.0 ** -8 if rounded else 0.0)


def flags(kind, B, T, rng):
    f = np.zeros((B, T), np.uint8)
    if kind == "all":
        f[:] = 1
    elif kind == "first":
        f[:, 0] = 1
    elif kind == "last":
        f[:, -1] = 1
    elif kind == "some":
        f[:] = rng.random((B, T)) < 0.05
        f *= rng.integers(1, 256, (B, T)).astype(np.uint8)      # any nonzero byte
    elif kind == "dense":
        f[:] = rng.random((B, T)) < 0.5
    else:
        assert kind == "none"
    return f


def longest(start):
    n = 0
    for row in start:
        at = np.concatenate([[0], np.flatnonzero(row), [len(row)]])
        n = max(n, int(np.diff(at).max()))
    return n


def inputs(dtype, B, T, d, kind, state=True, seed=0, rates=(1.0, 1e-3)):
    rng = np.random.default_rng(seed)
    dt = DT[dtype]

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dt)

    alpha = np.exp(rng.uniform(np.log(rates[1]), np.log(rates[0]), d)) * rng.choice([-1.0, 1.0], d)
    s = dict(x=normal(B, T, d), gates=normal(B, T, 2, d), alpha=torch.from_numpy(alpha.astype(np.float32)),
             start=torch.from_numpy(flags(kind, B, T, rng)), grad_h=normal(B, T, d))
    s["state"] = torch.from_numpy(rng.standard_normal((B, d), dtype=np.float32)) if state else None
    s["grad_state"] = torch.from_numpy(rng.standard_normal((B, d), dtype=np.float32)) if state else None
    return s


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def check(dtype, B, T, d, kind="some", state=True, seed=0, rates=(1.0, 1e-3)):
    announce("gated %s B=%d T=%d d=%d flags=%s state=%s seed=%d" % (dtype, B, T, d, kind, state, seed))
    s = inputs(dtype, B, T, d, kind, state, seed, rates)
    c = {k: None if v is None else v.to(DEV) for k, v in s.items()}
    h, last, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], final_state=True, keep_states=True)
    got = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    torch.cuda.synchronize()
    n = longest(s["start"].numpy())
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    rh, mh, rl, ml = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    assert h.dtype == DT[dtype] and last.dtype == kept.dtype == torch.float32
    e = cond_err(np64(h), rh, mh)
    assert e <= tol(dtype, n), ("h", e)
    e = cond_err(np64(last), rl, ml)
    assert e <= tol(dtype, n, rounded=False), ("state", e)
    want = np.concatenate([a["state"][:, None] if state else np.zeros((B, 1, d)), rh], 1)[:, :T:64]
    mag = np.concatenate([np.abs(want[:, :1]), mh], 1)[:, :T:64]
    e = cond_err(np64(kept), want, mag)
    assert e <= tol(dtype, n, rounded=False), ("states", e)
    w = ref.grads(a["x"], a["gates"], a["alpha"], a["start"], a["grad_h"], a["state"], a["grad_state"])
    for name, y in zip(("x", "gates", "alpha", "state"), got):
        assert y.dtype == (DT[dtype] if name in ("x", "gates") else torch.float32)
        e = cond_err(np64(y), *w[name])
        assert e <= tol(dtype, n, True, name in ("x", "gates")), ("d" + name, e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,d", [(1, 1, 1), (2, 5, 3), (1, 64, 64), (3, 65, 50), (2, 127, 64), (1, 128, 128), (2, 129, 66),
                                   (1, 255, 7), (2, 257, 63), (1, 1000, 256), (5, 333, 250), (64, 1, 256), (2, 2050, 33),
                                   (1, 4097, 8), (300, 3, 5)])
def test_sizes(dtype, B, T, d):
    check(dtype, B, T, d, seed=B + T + d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "all", "first", "last", "dense"])
@pytest.mark.parametrize("state", [False, True])
def test_flags(dtype, kind, state):
    check(dtype, 3, 700, 68, kind, state, seed=11)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rates", [(50.0, 0.3), (0.6, 0.4), (1e-3, 1e-6), (0.49, 1e-2)])
def test_rates(dtype, rates):
    check(dtype, 2, 600, 64, "some", True, 5, rates)


def test_nothing_to_do():
    """No tapes, no steps, no features: a carried state and its gradient pass through."""
    announce("gated empty")
    for B, T, d in ((0, 5, 8), (2, 0, 8), (2, 5, 0), (0, 0, 0)):
        x, gates = torch.zeros(B, T, d, device=DEV, requires_grad=True), torch.zeros(B, T, 2, d, device=DEV, requires_grad=True)
        alpha, start = torch.ones(d, device=DEV, requires_grad=True), torch.zeros(B, T, dtype=torch.uint8, device=DEV)
        state = torch.randn(B, d, device=DEV).requires_grad_(True)
        h, last = mb.gated_scan(x, gates, alpha, start, state, final_state=True)
        assert h.shape == (B, T, d) and torch.equal(last, state)
        up = torch.randn(B, d, device=DEV)
        dx, dg, da, ds = torch.autograd.grad((h, last), (x, gates, alpha, state), (torch.zeros_like(h), up))
        assert dx.shape == x.shape and dg.shape == gates.shape and not bool(da.any()) and torch.equal(ds, up)
        if T == 0:
            assert not bool(mb.gated_scan(x, gates, alpha, start, final_state=True)[1].any())
    assert mb.gated_step(torch.zeros(0, 8, device=DEV), torch.zeros(0, 2, 8, device=DEV), torch.ones(8, device=DEV),
                         torch.zeros(0, 8, device=DEV)).shape == (0, 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,d", [(1, 3, 1 << 18), (1, 70, (1 << 18) - 1), (6000, 70, 2), (1, 20000, 3)])
def test_wide_and_many(dtype, B, T, d):
    """The widest rows, many tapes, many tiles of one chain."""
    check(dtype, B, T, d, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,d", [(61, 4, 688), (5, 31, 70), (5, 32, 65), (5, 33, 64), (2, 63, 130), (9, 64, 129), (2, 66, 3)])
def test_short_tapes(dtype, B, T, d):
    """Tapes around the sizes where the tiles change."""
    check(dtype, B, T, d, seed=T)
    check(dtype, B, T, d, "none", seed=T + 1)


@pytest.mark.parametrize("need", [(0,), (1,), (2,), (3,), (0, 3)])
def test_some_gradients(need):
    """Whichever inputs want a gradient, it is the one that all of them get; outputs that
    nothing hangs on count as zero."""
    announce("gated need=%s" % (need,))
    s = {k: v.to(DEV) for k, v in inputs("f32", 2, 300, 64, "some", seed=3).items()}
    names = ("x", "gates", "alpha", "state")

    def run(need, grad_h, grad_state):
        leaves = [s[k].detach().requires_grad_(j in need) for j, k in enumerate(names)]
        h, last = mb.gated_scan(*leaves[:3], s["start"], leaves[3], final_state=True)
        outs, ups = zip(*[(o, g) for o, g in ((h, grad_h), (last, grad_state)) if g is not None])
        return dict(zip(need, torch.autograd.grad(outs, [leaves[j] for j in need], ups)))

    zh, zs = torch.zeros_like(s["grad_h"]), torch.zeros_like(s["grad_state"])
    for gh, gs in ((s["grad_h"], s["grad_state"]), (s["grad_h"], None), (None, s["grad_state"])):
        whole = run((0, 1, 2, 3), zh if gh is None else gh, zs if gs is None else gs)
        for j, g in run(need, gh, gs).items():
            assert torch.equal(g, whole[j])


@pytest.mark.parametrize("T", [600, 1300])
def test_one_begin_anywhere(T):
    """A begin step at each place of its own tape, around the edges of lanes and tiles."""
    announce("gated one begin T=%d" % T)
    at = sorted({t for e in range(0, T, 64) for t in (e - 1, e, e + 1) if 0 <= t < T} | {T - 1})
    s = inputs("f32", len(at), T, 8, "none", True, T)
    s["start"] = torch.zeros(len(at), T, dtype=torch.uint8)
    s["start"][torch.arange(len(at)), torch.tensor(at)] = 1
    c = {k: v.to(DEV) for k, v in s.items()}
    h, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
    got = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    rh, mh, _, _ = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    assert cond_err(np64(h), rh, mh) <= tol("f32", T)
    w = ref.grads(a["x"], a["gates"], a["alpha"], a["start"], a["grad_h"], a["state"], a["grad_state"])
    for name, y in zip(("x", "gates", "alpha", "state"), got):
        assert cond_err(np64(y), *w[name]) <= tol("f32", T, True), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("alpha", [2e-2, 1e-3, 1e-5])
def test_gates_that_stand_still(dtype, alpha):
    """Constant gates and input: h_t = b (1 - a^(t+1)) / (1 - a).  One rounded a would
    be off the same way at every step, 2^-25 / (1 - a) of a long memory, 3e-3 at 1e-5."""
    T = 30000
    announce("gated constant %s alpha=%g" % (dtype, alpha))
    x = torch.ones(1, T, 4, device=DEV, dtype=DT[dtype])
    gates = torch.zeros(1, T, 2, 4, device=DEV, dtype=DT[dtype])
    start = torch.zeros(1, T, dtype=torch.uint8, device=DEV)
    al = torch.full((4,), alpha, device=DEV)
    h, last = mb.scan_gated(x, gates, al, start, final_state=True)
    u = 0.5 * float(al[0])
    b = np.sqrt(-np.expm1(-2 * u)) * 0.5
    want = b * -np.expm1(-u * np.arange(1, T + 1)) / -np.expm1(-u)
    # the state's roundings may all go the same way here: two a step in a run of up to 16, two
    # for each of a tile's 16 runs, two a tile of 64 steps or more
    bound = (32 + 11 + 2 * (16 + 16 + T / 64)) * E * (2 if dtype == "bf16" else 1)
    assert float(np.abs(np64(last)[0] / want[-1] - 1).max()) <= bound
    assert np.abs(np64(h)[0] / want[:, None] - 1).max() <= bound + (2.0 ** -8 if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_gates_and_zero_rate(dtype):
    announce("gated infinite gates %s" % dtype)
    s = inputs(dtype, 2, 300, 16, "none", True, 3)
    s["gates"][0, 40:80, 0] = -float("inf")          # holds
    s["gates"][0, 100:120, 0] = float("inf")         # whole rate
    s["gates"][1, 10:200, 1] = -float("inf")         # lets nothing in
    s["gates"][1, 220:240, 1] = float("inf")
    s["alpha"][3] = 0.0
    c = {k: v.to(DEV) for k, v in s.items()}
    h, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
    assert bool((h[:, :, 3] == c["state"][:, None, 3].to(h.dtype)).all())
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    rh, mh, _, _ = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    assert cond_err(np64(h), rh, mh) <= tol(dtype, 300)
    # what holds is one number, reached along different sums on the two sides of a run's edge:
    # each is off by at most the bound above
    assert cond_err(np64(h[0, 40:80]), np64(h[0, 39:40]), mh[0, 39:40]) <= 2 * tol(dtype, 300)
    got = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    w = ref.grads(a["x"], a["gates"], a["alpha"], a["start"], a["grad_h"], a["state"], a["grad_state"])
    for name, y in zip(("x", "gates", "alpha", "state"), got):
        assert cond_err(np64(y), *w[name]) <= tol(dtype, 300, True, name in ("x", "gates")), name
    assert float(got[2][3]) == 0.0


@pytest.mark.parametrize("what,bad", [(w, float("nan")) for w in "xrig"] + [(w, float("inf")) for w in "xg"])
def test_bad_values_stay_in_their_episode(what, bad):
    announce("gated %s = %s" % (what, bad))
    T, d = 900, 20
    s = inputs("f32", 1, T, d, "none", True, 1)
    for t in (300, 600):
        s["start"][0, t] = 1
    at = {"x": s["x"][0, 400], "r": s["gates"][0, 400, 0], "i": s["gates"][0, 400, 1], "g": s["grad_h"][0, 400]}[what]
    at[7] = bad
    c = {k: v.to(DEV) for k, v in s.items()}
    h, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
    gx, gg, ga, gs = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    ok = torch.isfinite(h)[0]
    ok[400:600, 7] = True
    assert bool(ok.all()), "h"
    if what != "g":
        assert not bool(torch.isfinite(h[0, 400:600, 7]).any())
    for t in (gx[0], gg[0, :, 0], gg[0, :, 1]):
        ok = torch.isfinite(t)
        ok[300:600, 7] = True
        assert bool(ok.all())
    assert bool(torch.isfinite(gs).all())
    ok = torch.isfinite(ga)
    ok[7] = True
    assert bool(ok.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_runs_are_equal(dtype):
    """The tiles' order of arrival changes nothing."""
    announce("gated equal runs %s" % dtype)
    s = inputs(dtype, 2, 9000, 130, "none", True, 9)
    c = {k: v.to(DEV) for k, v in s.items()}
    first = None
    for _ in range(6):
        got = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], final_state=True, keep_states=True)
        got += mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], got[2], c["grad_h"], c["grad_state"])
        if first is None:
            first = [t.clone() for t in got]
        assert all(torch.equal(x, y) for x, y in zip(first, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cut", [1, 128, 500, 999])
def test_carried_state(dtype, cut):
    announce("gated carried state %s cut=%d" % (dtype, cut))
    s = inputs(dtype, 2, 1000, 40, "some", True, cut)
    c = {k: v.to(DEV) for k, v in s.items()}
    whole, end = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], final_state=True)
    parts, state = [], c["state"]
    for lo, hi in ((0, cut), (cut, 1000)):
        h, state = mb.scan_gated(c["x"][:, lo:hi].contiguous(), c["gates"][:, lo:hi].contiguous(), c["alpha"],
                                 c["start"][:, lo:hi].contiguous(), state, final_state=True)
        parts.append(h)
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    _, mh, _, ml = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    assert cond_err(np64(torch.cat(parts, 1)), np64(whole), mh) <= 2 * tol(dtype, 1000)
    assert cond_err(np64(state), np64(end), ml) <= 2 * tol(dtype, 1000, rounded=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,d", [(1, 1), (3, 50), (16, 256), (257, 33), (5, 4096)])
def test_step(dtype, B, d):
    announce("gated step %s B=%d d=%d" % (dtype, B, d))
    T = 7
    s = inputs(dtype, B, T, d, "dense", True, B + d)
    c = {k: v.to(DEV) for k, v in s.items()}
    state = c["state"].clone()
    out = [mb.gated_step(c["x"][:, t].contiguous(), c["gates"][:, t].contiguous(), c["alpha"], state,
                         c["start"][:, t].contiguous()) for t in range(T)]
    a = {k: np64(v) if k != "start" else v.numpy() for k, v in s.items()}
    rh, mh, rl, ml = ref.scan(a["x"], a["gates"], a["alpha"], a["start"], a["state"])
    assert cond_err(np64(torch.stack(out, 1)), rh, mh) <= tol(dtype, T)
    assert cond_err(np64(state), rl, ml) <= tol(dtype, T, rounded=False)
    # no flags: nobody begins
    state = c["state"].clone()
    h = mb.gated_step(c["x"][:, 0].contiguous(), c["gates"][:, 0].contiguous(), c["alpha"], state)
    rh, mh, _, _ = ref.scan(a["x"][:, :1], a["gates"][:, :1], a["alpha"], np.zeros((B, 1), np.uint8), a["state"])
    assert cond_err(np64(h), rh[:, 0], mh[:, 0]) <= tol(dtype, 1)


def test_step_that_begins_forgets_a_nan():
    announce("gated step nan")
    state = torch.full((2, 8), float("nan"), device=DEV)
    x, gates, alpha = torch.ones(2, 8, device=DEV), torch.zeros(2, 2, 8, device=DEV), torch.full((8,), 0.1, device=DEV)
    h = mb.gated_step(x, gates, alpha, state, torch.tensor([1, 0], dtype=torch.uint8, device=DEV))
    assert bool(torch.isfinite(h[0]).all()) and not bool(torch.isfinite(h[1]).any())


def test_step_bumps_the_state():
    announce("gated step version")
    state = torch.zeros(1, 4, device=DEV)
    leaf = torch.ones(1, 4, device=DEV, requires_grad=True)
    y = (leaf * state).sum()
    with torch.no_grad():
        mb.gated_step(torch.ones(1, 4, device=DEV), torch.zeros(1, 2, 4, device=DEV), torch.ones(4, device=DEV), state)
    with pytest.raises(RuntimeError):
        y.backward()
    with pytest.raises(RuntimeError):
        mb.gated_step(leaf, torch.zeros(1, 2, 4, device=DEV), torch.ones(4, device=DEV), state)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_autograd(dtype):
    announce("gated autograd %s" % dtype)
    s = inputs(dtype, 2, 300, 24, "some", True, 2)
    c = {k: v.to(DEV) for k, v in s.items()}
    leaves = [c[k].clone().requires_grad_(True) for k in ("x", "gates", "alpha", "state")]
    h, last = mb.gated_scan(*leaves[:3], c["start"], leaves[3], final_state=True)
    torch.autograd.backward((h, last), (c["grad_h"], c["grad_state"]))
    _, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
    want = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])
    for x, y in zip(leaves, want):
        assert torch.equal(x.grad, y)
    # gradients that are views, one output alone, some inputs alone
    h = mb.gated_scan(*leaves[:3], c["start"])
    gx, = torch.autograd.grad(h.float().sum(), leaves[:1])
    _, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], keep_states=True)
    want = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, torch.ones_like(c["x"]))
    assert torch.equal(gx, want[0])
    h, last = mb.gated_scan(*leaves[:3], c["start"], leaves[3], final_state=True)
    ga, = torch.autograd.grad(last, leaves[2:3], c["grad_state"])
    want = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept * 0 + mb.scan_gated(
        c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)[1], torch.zeros_like(c["x"]), c["grad_state"])
    assert torch.equal(ga, want[2])
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(mb.gated_scan(*leaves[:3], c["start"]).float().sum(), leaves[:1], create_graph=True)
        g.float().sum().backward()


def test_differences():
    """Directional derivative of a weighted sum of h, by central differences: with steps
    of 2^-6 the third derivative leaves about 1e-4 of it, the fp32 sums about 1e-5."""
    announce("gated differences")
    s = inputs("f32", 2, 200, 12, "some", True, 4, rates=(1.0, 0.05))
    c = {k: v.to(DEV) for k, v in s.items()}
    names = ("x", "gates", "alpha", "state")
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    v = {k: torch.randn(c[k].shape, generator=g, device=DEV) * (0.05 * c[k].abs() if k == "alpha" else 1.0) for k in names}

    def value(t):
        h = mb.scan_gated(*(c[k] + t * v[k] for k in names[:3]), c["start"], c["state"] + t * v["state"])
        return float((h.double() * c["grad_h"].double()).sum())

    eps = 2.0 ** -6
    want = (8 * (value(eps) - value(-eps)) - (value(2 * eps) - value(-2 * eps))) / (12 * eps)
    _, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
    got = mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"])
    terms = [float((y.double() * v[k].double()).sum()) for k, y in zip(names, got)]
    assert abs(sum(terms) - want) <= 1e-3 * sum(abs(t) for t in terms), (terms, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_odd_addresses_and_nothing_behind(dtype):
    """Operands that start one element into their memory, outputs with guards around."""
    announce("gated guards %s" % dtype)
    B, T, d = 2, 131, 37
    s = inputs(dtype, B, T, d, "some", True, 6)
    want = mb.scan_gated(*(s[k].to(DEV) for k in ("x", "gates", "alpha", "start", "state")), final_state=True,
                         keep_states=True)
    dwant = mb.scan_gated_bwd(*(s[k].to(DEV) for k in ("x", "gates", "alpha", "start")), want[2], s["grad_h"].to(DEV),
                              s["grad_state"].to(DEV))

    def shifted(t):
        buf = torch.full((t.numel() + 130,), 7, dtype=t.dtype, device=DEV)
        view = buf[65:65 + t.numel()].view(t.shape)
        view.copy_(t)
        return buf, view

    ins = {k: shifted(s[k])[1] for k in s}
    outs = [shifted(torch.zeros_like(t)) for t in want + dwant]
    o = [v.data_ptr() for _, v in outs]
    dt = mb.F32 if dtype == "f32" else mb.BF16
    n = max(mb.memoroid_scan_gated_workspace_bytes(B, T, d, dt), mb.memoroid_scan_gated_bwd_workspace_bytes(B, T, d, dt))
    ws = torch.randint(0, 256, (n + 512,), dtype=torch.uint8, device=DEV)
    keep = ws[n:].clone()
    st = torch.cuda.current_stream().cuda_stream
    p = {k: v.data_ptr() for k, v in ins.items()}
    assert mb.memoroid_scan_gated(p["x"], p["gates"], p["alpha"], p["start"], p["state"], o[0], o[1], o[2], B, T, d, dt,
                                  ws.data_ptr(), n, st) == mb.OK
    assert mb.workspace_status(ws) == mb.OK
    assert mb.memoroid_scan_gated_bwd(p["x"], p["gates"], p["alpha"], p["start"], o[2], p["grad_h"], p["grad_state"], o[3],
                                      o[4], o[5], o[6], B, T, d, dt, ws.data_ptr(), n, st) == mb.OK
    assert mb.workspace_status(ws) == mb.OK
    for (buf, view), w in zip(outs, want + dwant):
        assert torch.equal(view, w)
        assert bool((buf[:65] == 7).all()) and bool((buf[65 + w.numel():] == 7).all())
    assert torch.equal(ws[n:], keep)


def test_past_32_bits():
    """More than 2^31 values in h, 2^32 in the gates: the last tape is what it is alone."""
    announce("gated past 2^31 values")
    B, T, d = 9, 65536, 4096
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn(1, T, d, device=DEV, generator=g).to(torch.bfloat16)
    gates = torch.randn(1, T, 2, d, device=DEV, generator=g).to(torch.bfloat16)
    alpha = torch.rand(d, device=DEV, generator=g) * 0.1
    start = (torch.rand(1, T, device=DEV, generator=g) < 0.001).to(torch.uint8)
    want, kept = mb.scan_gated(x, gates, alpha, start, keep_states=True)
    dwant = mb.scan_gated_bwd(x, gates, alpha, start, kept, x)
    bx, bg, bs = torch.zeros(B, T, d, device=DEV, dtype=torch.bfloat16), torch.zeros(B, T, 2, d, device=DEV, dtype=torch.bfloat16), \
        torch.zeros(B, T, device=DEV, dtype=torch.uint8)
    bx[-1], bg[-1], bs[-1] = x[0], gates[0], start[0]
    h, kept = mb.scan_gated(bx, bg, alpha, bs, keep_states=True)
    assert torch.equal(h[-1], want[0])
    assert not bool(h[0].any())
    got = mb.scan_gated_bwd(bx, bg, alpha, bs, kept, bx)
    for y, w in zip(got[:2], dwant[:2]):
        assert torch.equal(y[-1], w[0])
        assert not bool(y[0].any())


def test_streams():
    """Calls on two streams at once, each with a workspace of its own."""
    announce("gated streams")
    s = inputs("f32", 2, 4000, 64, "none", True, 8)
    c = {k: v.to(DEV) for k, v in s.items()}

    def both():
        h, kept = mb.scan_gated(c["x"], c["gates"], c["alpha"], c["start"], c["state"], keep_states=True)
        return (h,) + mb.scan_gated_bwd(c["x"], c["gates"], c["alpha"], c["start"], kept, c["grad_h"], c["grad_state"])

    want = both()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(both())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))
