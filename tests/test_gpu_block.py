"""Layer norm, gated recurrence and dropout together, as a residual block runs them:
training against the block in 64 bits through autograd, generating step by step, and
captured in a graph."""
import numpy as np
import pytest

import gated_ref as ref
from conftest import announce

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SEED, P = 77, 0.1


def make(dtype, B, T, d, e, seed=0):
    """Two blocks' parameters (model width d, inner width e), inputs and flags."""
    rng = np.random.default_rng(seed)

    def normal(*shape, scale=1.0):
        return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32))

    blocks = [dict(w=1 + 0.1 * normal(d), b=0.1 * normal(d), into=normal(d, 3 * e, scale=d ** -0.5),
                   out=normal(e, d, scale=e ** -0.5), alpha=torch.from_numpy(rng.uniform(1e-3, 1.0, e).astype(np.float32)))
              for _ in range(2)]
    start = torch.from_numpy((rng.random((B, T)) < 0.02).astype(np.uint8))
    return blocks, normal(B, T, d).to(dtype), start, normal(B, e)


def block_own(x, s, k, start, rng, site, state, p, steps=False):
    """x: the previous block's output before dropout; s: the residual stream."""
    y, s = mb.layer_norm(x, k["w"], k["b"], residual=s, p=p, rng=rng, site=site)
    z = y @ k["into"].to(y.dtype)
    e = k["alpha"].numel()
    u, gates = z[..., :e].contiguous(), z[..., e:].reshape(z.shape[:-1] + (2, e)).contiguous()
    h = mb.gated_step(u, gates, k["alpha"], state, start) if steps else mb.gated_scan(u, gates, k["alpha"], start, state)
    return h @ k["out"].to(y.dtype), s


def model_own(blocks, x, start, rng, states, p=P):
    s, o = torch.zeros_like(x), x
    for i, k in enumerate(blocks):
        o, s = block_own(o, s, k, start, rng, i, states[i], p)
    return mb.dropout(o, p, rng, len(blocks), residual=s)


def keep(shape, step, site):
    rows = shape[0] * shape[1]
    return torch.from_numpy(ref.keep(P, SEED, step, site, rows, shape[2])).reshape(shape).double() / (1 - P)


def model_64(blocks, x, start, step, states):
    s, o = torch.zeros_like(x), x
    for i, k in enumerate(blocks):
        s = s + o * keep(x.shape, step, i)
        c = s - s.mean(-1, keepdim=True)
        y = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * k["w"] + k["b"]
        z = y @ k["into"]
        e = k["alpha"].numel()
        a = torch.exp(-k["alpha"].abs() * torch.sigmoid(z[..., e:2 * e]))
        b = torch.sqrt(1 - a * a) * torch.sigmoid(z[..., 2 * e:]) * z[..., :e]
        h, hs = states[i], []
        for t in range(x.shape[1]):
            h = torch.where(start[:, t, None] != 0, b[:, t], a[:, t] * h + b[:, t])
            hs.append(h)
        o = torch.stack(hs, 1) @ k["out"]
    return s + o * keep(x.shape, step, len(blocks))


def leaves_of(blocks, to):
    return [{n: to(v).requires_grad_(True) for n, v in k.items()} for k in blocks]


def far(got, want):
    """Largest error over the largest value."""
    want = want.detach()
    return float((got.detach().double().cpu() - want).abs().max() / want.abs().max())


def test_training():
    """fp32 blocks against 64 bits.  A relative 2^-24 times the roundings on the way: two
    norms (240), two recurrences (72 + 8 sqrt 150 = 170) and four projections of up to 96
    terms (torch's own fp32 products, 96) each way make at most 2000, 1.2e-4."""
    announce("block training f32")
    blocks, x, start, state = make(torch.float32, 3, 150, 32, 48)
    rng = torch.tensor([SEED, 5], dtype=torch.int64, device=DEV)
    mine = leaves_of(blocks, lambda v: v.to(DEV))
    xs = x.to(DEV).requires_grad_(True)
    st = [state.to(DEV).requires_grad_(True) for _ in blocks]
    y = model_own(mine, xs, start.to(DEV), rng, st)
    r = torch.randn(y.shape, generator=torch.Generator().manual_seed(1))
    (y * r.to(DEV)).sum().backward()
    theirs = leaves_of(blocks, lambda v: v.double())
    xd = x.double().requires_grad_(True)
    sd = [state.double().requires_grad_(True) for _ in blocks]
    want = model_64(theirs, xd, start, 5, sd)
    (want * r.double()).sum().backward()
    assert far(y, want) <= 1.2e-4
    assert far(xs.grad, xd.grad) <= 1.2e-4
    for a, b in zip(st, sd):
        assert far(a.grad, b.grad) <= 1.2e-4
    for a, b in zip(mine, theirs):
        for n in a:
            assert far(a[n].grad, b[n].grad) <= 1.2e-4, n


def test_generating():
    """Reading a prompt at once and then going on step by step gives what the whole tape
    gives (each as far from 64 bits as above, without dropout)."""
    announce("block generating f32")
    blocks, x, start, state = make(torch.float32, 4, 60, 32, 48, seed=2)
    dev = [{n: v.to(DEV) for n, v in k.items()} for k in blocks]
    xs, st = x.to(DEV), start.to(DEV)
    with torch.no_grad():
        want = model_own(dev, xs, st, None, [state.to(DEV)] * 2, p=0.0)
        states, s, o = [], torch.zeros_like(xs[:, :40]), xs[:, :40].contiguous()
        for k in dev:
            y, s = mb.norm_rows(o, k["w"], k["b"], residual=s)
            z = y @ k["into"]
            u, gates = z[..., :48].contiguous(), z[..., 48:].reshape(4, 40, 2, 48).contiguous()
            h, last = mb.scan_gated(u, gates, k["alpha"], st[:, :40].contiguous(), state.to(DEV), final_state=True)
            states.append(last)
            o = h @ k["out"]
        assert far(mb.drop_rows(o, 0.0, None, residual=s), want[:, :40].double().cpu()) <= 1.2e-4
        for t in range(40, 60):
            s, o = torch.zeros(4, 32, device=DEV), xs[:, t].contiguous()
            for i, k in enumerate(dev):
                o, s = block_own(o, s, k, st[:, t].contiguous(), None, i, states[i], 0.0, steps=True)
            assert far(o + s, want[:, t].double().cpu()) <= 2.4e-4


def raw_pass(c, rng):
    """Forward and gradient of norm, recurrence and dropout through the raw calls."""
    y, s, st = mb.norm_rows(c["x"], c["w"], c["b"], residual=c["res"], p=P, rng=rng, site=1, keep_stats=True)
    h, last, kept = mb.scan_gated(y, c["gates"], c["alpha"], c["start"], c["state"], final_state=True, keep_states=True)
    out = mb.drop_rows(h, P, rng, 2, s)
    gh = mb.drop_rows(c["g"], P, rng, 2)
    gy, gg, ga, gs = mb.scan_gated_bwd(y, c["gates"], c["alpha"], c["start"], kept, gh, last)
    return (out, last, gg, ga, gs) + tuple(mb.norm_rows_bwd(c["x"], st, gy, c["w"], c["res"], c["g"], P, rng, 1))


def raw_inputs(dtype, B, T, d, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, dt=dtype):
        return torch.randn(shape, generator=g, device=DEV).to(dt)

    return dict(x=normal(B, T, d), res=normal(B, T, d), g=normal(B, T, d), gates=normal(B, T, 2, d),
                w=normal(d, dt=torch.float32), b=normal(d, dt=torch.float32), alpha=normal(d, dt=torch.float32) * 0.1,
                state=normal(B, d, dt=torch.float32), start=(torch.rand(B, T, generator=g, device=DEV) < 0.01).to(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,d", [(2, 3000, 64), (3, 70, 50)])
def test_captured(dtype, B, T, d):
    """A captured pass, its inputs and the step of its dropout changed between replays,
    with eager work between them, against the eager pass on the same inputs; and two
    graphs replayed on two streams at once."""
    announce("block captured %s %d %d %d" % (dtype, B, T, d))
    side = torch.cuda.Stream()
    sets = []
    for seed in (0, 1):
        c, rng = raw_inputs(dtype, B, T, d, seed), torch.tensor([seed, 0], dtype=torch.int64, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            raw_pass(c, rng)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = raw_pass(c, rng)
        sets.append((c, rng, graph, out))
    for turn in range(5):
        c, rng, graph, out = sets[0]
        fresh = raw_inputs(dtype, B, T, d, 10 + turn)
        for k in c:
            c[k].copy_(fresh[k])
        rng[1] += 1
        graph.replay()
        want = raw_pass(c, rng)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), turn
    want = [raw_pass(c, rng) for c, rng, _, _ in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for st, (_, _, graph, _) in zip(streams, sets):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for (_, _, _, out), w in zip(sets, want):
        assert all(torch.equal(x, y) for x, y in zip(out, w))


def test_captured_training():
    """A whole training pass through autograd in a graph, on leaves of its own."""
    announce("block captured training")
    blocks, x, start, state = make(torch.float32, 2, 90, 32, 48, seed=4)
    rng = torch.tensor([SEED, 0], dtype=torch.int64, device=DEV)
    xs, st, s0 = x.to(DEV), start.to(DEV), state.to(DEV)
    mine = leaves_of(blocks, lambda v: v.to(DEV))
    params = [v for k in mine for v in k.values()]

    def grads():
        return torch.autograd.grad(model_own(mine, xs, st, rng, [s0, s0]).square().mean(), params)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            grads()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads()
    for turn in range(4):
        rng[1] += 1
        graph.replay()
        want = grads()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert far(a, b.double().cpu()) <= 1e-5, turn


# ------------------------------------------------------------- autograd nodes

def test_refused_by_the_library():
    """What the library refuses is a MemoroidError with its status, as from the raw forms."""
    announce("nodes refused")
    x = torch.zeros(1, 16385, device=DEV, requires_grad=True)
    for f in (lambda: mb.layer_norm(x), lambda: mb.norm_rows(x)):
        with pytest.raises(mb.MemoroidError) as e:
            f()
        assert e.value.status == mb.EUNSUPPORTED and "memoroid_layer_norm failed" in str(e.value)
    d = (1 << 18) + 1
    with pytest.raises(mb.MemoroidError) as e:
        mb.gated_scan(torch.zeros(1, 1, d, device=DEV), torch.zeros(1, 1, 2, d, device=DEV), torch.zeros(d, device=DEV),
                      torch.zeros(1, 1, dtype=torch.uint8, device=DEV))
    assert e.value.status == mb.EUNSUPPORTED
    with pytest.raises(mb.MemoroidError):
        mb.layer_norm(x[:, :8].detach(), eps=-1.0)


def test_workspaces():
    """The caller's workspace, whatever it holds; one that is too small is not used, one with
    gaps or on the host is refused."""
    announce("nodes workspaces")
    torch.manual_seed(1)
    x, gates = torch.randn(2, 400, 40, device=DEV), torch.randn(2, 400, 2, 40, device=DEV)
    alpha, start = torch.rand(40, device=DEV), torch.zeros(2, 400, dtype=torch.uint8, device=DEV)
    h, kept = mb.scan_gated(x, gates, alpha, start, keep_states=True)
    want = mb.scan_gated_bwd(x, gates, alpha, start, kept, h)
    y, st = mb.norm_rows(x, alpha, keep_stats=True)
    rows = mb.norm_rows_bwd(x, st, h, alpha)
    for fill in (0, 255, 7):
        ws = torch.full((1 << 20,), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(mb.scan_gated(x, gates, alpha, start, workspace=ws), h)
        assert mb.workspace_status(ws) == mb.OK
        for a, b in zip(mb.scan_gated_bwd(x, gates, alpha, start, kept, h, workspace=ws), want):
            assert torch.equal(a, b)
        assert mb.workspace_status(ws) == mb.OK
        for a, b in zip(mb.norm_rows_bwd(x, st, h, alpha, workspace=ws), rows):
            assert (a is None and b is None) or torch.equal(a, b)
    small = torch.full((300,), 9, dtype=torch.uint8, device=DEV)
    assert torch.equal(mb.scan_gated(x, gates, alpha, start, workspace=small), h)
    assert bool((small == 9).all())
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 21, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(ValueError):
            mb.scan_gated(x, gates, alpha, start, workspace=ws)
        with pytest.raises(ValueError):
            mb.scan_gated_bwd(x, gates, alpha, start, kept, h, workspace=ws)
        with pytest.raises(ValueError):
            mb.norm_rows_bwd(x, st, h, alpha, workspace=ws)


def test_out_of_memory():
    """No memory for an output is torch's error for it, and the call can be made again."""
    announce("nodes out of memory")
    x = torch.zeros(1 << 18, 1 << 10, device=DEV)
    rng = torch.tensor([SEED, 1], dtype=torch.int64, device=DEV)
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (1 << 28)) / total)
    try:
        for f in (lambda: mb.drop_rows(x, 0.5, rng), lambda: mb.dropout(x, 0.5, rng), lambda: mb.layer_norm(x)):
            with pytest.raises(torch.OutOfMemoryError):
                f()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert torch.equal(mb.drop_rows(x, 0.5, rng), x)


@pytest.mark.parametrize("given", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("residual", [False, True])
def test_wanted_gradients_of_the_norm(given, residual):
    """Any of the inputs given, any of those wanting a gradient: each the raw form's."""
    announce("nodes norm %s %s" % (given, residual))
    torch.manual_seed(0)
    x, gy, gs, res = (torch.randn(7, 40, device=DEV) for _ in range(4))
    w, b = (torch.randn(40, device=DEV) if g else None for g in given)
    res = res if residual else None
    rng = torch.tensor([SEED, 1], dtype=torch.int64, device=DEV)
    *_, st = mb.norm_rows(x, w, b, residual=res, p=0.2, rng=rng, keep_stats=True)
    raw = mb.norm_rows_bwd(x, st, gy, w, res, gs, 0.2, rng)
    want = dict(zip("xrwb", raw))
    names = [n for n, v in zip("xrwb", (x, res, w, b)) if v is not None]
    for mask in range(1, 1 << len(names)):
        leaves = {n: v.detach().requires_grad_(n in names and bool(mask >> names.index(n) & 1))
                  for n, v in zip("xrwb", (x, res, w, b)) if v is not None}
        y, s = mb.layer_norm(leaves["x"], leaves.get("w"), leaves.get("b"), residual=leaves.get("r"), p=0.2, rng=rng)
        wanted = [n for n in names if leaves[n].requires_grad]
        for n, g in zip(wanted, torch.autograd.grad((y, s), [leaves[n] for n in wanted], (gy, gs))):
            assert g.dtype == torch.float32 and torch.equal(g, want[n]), (mask, n)


def test_nodes_once_and_unchanged():
    """No second derivative, also where only one output's gradient is in the graph; inputs
    that changed after the forward pass are refused; under no_grad there is no node."""
    announce("nodes once")
    x = torch.randn(2, 9, 16, device=DEV).requires_grad_(True)
    gates, alpha = torch.randn(2, 9, 2, 16, device=DEV), torch.rand(16, device=DEV)
    start = torch.zeros(2, 9, dtype=torch.uint8, device=DEV)
    rng = torch.tensor([SEED, 1], dtype=torch.int64, device=DEV)
    forms = (lambda v: mb.gated_scan(v, gates, alpha, start), lambda v: mb.layer_norm(v), lambda v: mb.dropout(v, 0.3, rng))
    for f in forms:
        first, = torch.autograd.grad(f(x).square().sum(), x)
        g, = torch.autograd.grad(f(x).square().sum(), x, create_graph=True)
        assert torch.equal(g, first) and g.requires_grad
        with pytest.raises(RuntimeError, match="twice"):
            g.sum().backward()
        with torch.no_grad():
            y = f(x)
        assert not y.requires_grad and torch.equal(y, f(x))
    for f in forms[:2]:
        v = x.detach().clone().requires_grad_(True)
        u = v * 1.0
        y = f(u)
        with torch.no_grad():
            u.add_(1.0)
        with pytest.raises(RuntimeError, match="inplace"):
            y.sum().backward()


def test_nodes_on_threads_and_streams():
    """Two threads, a stream each, train at once: the results of one alone."""
    announce("nodes threads")
    import threading

    def work(seed, out, turns):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            x, up = (torch.randn(2, 3000, 64, device=DEV, generator=g) for _ in range(2))
            gates = torch.randn(2, 3000, 2, 64, device=DEV, generator=g)
            alpha = torch.rand(64, device=DEV, generator=g).mul_(0.1).requires_grad_(True)
            start = torch.zeros(2, 3000, dtype=torch.uint8, device=DEV)
            rng = torch.tensor([seed, 1], dtype=torch.int64, device=DEV)
            w = torch.ones(64, device=DEV, requires_grad=True)
            x.requires_grad_(True)
            for _ in range(turns):
                y, s = mb.layer_norm(x, w, residual=up, p=0.1, rng=rng)
                h = mb.dropout(mb.gated_scan(y, gates, alpha, start), 0.1, rng, 1, s)
                got = torch.autograd.grad(h, (x, w, alpha), up)
            out[seed] = [t.detach().clone() for t in (h, *got)]
            stream.synchronize()

    alone, both = {}, {}
    for seed in (1, 2):
        work(seed, alone, 1)
    threads = [threading.Thread(target=work, args=(seed, both, 20)) for seed in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert sorted(both) == [1, 2]
    for seed in (1, 2):
        assert all(torch.equal(a, b) for a, b in zip(alone[seed], both[seed]))
