"""Norms and rotation of queries and keys on the GPU against rotate_ref.py, error
relative to max(|r|, m).

Tolerances.  fp32: a row's sum of 128 squares (12 roundings in a row of sums, half
of them in its root), the root's and the sine's few, the angle's 2^-24 turns (pi
2^-23 of the partner), four products: below 32 2^-24 = 2e-6.  The gradient goes
through a second sum of the row and a cube of the root: 4e-6; the weights' sums
add 64 rows at most to a lane, 4e-6 more.  bf16: the rounding of the result,
2^-8, and the same."""
import numpy as np
import pytest

import rotate_ref as ref
from conftest import announce, cond_err

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def check(dtype, B, T, H, Hk, d, rot, inter, norm=(True, True), eps=1e-6, amp=1.0, far=0, seed=0):
    announce("rotate %s B=%d T=%d H=%d/%d d=%d rot=%d inter=%d norm=%s far=%d" % (dtype, B, T, H, Hk, d, rot, inter, norm, far))
    rng = np.random.default_rng(seed)
    dt = DT[dtype]

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dt)

    q, gq = normal(B, T, H, d), normal(B, T, H, d)
    k, gk = (normal(B, T, Hk, d), normal(B, T, Hk, d)) if Hk else (None, None)
    wq, wk = (torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)) if n else None for n in norm)
    if not Hk:
        wk = None
    pos = torch.from_numpy((far + rng.integers(0, 5000, (B, T))).astype(np.int32))
    freq = mb.rotary_frequencies(rot) if rot else None
    dev = [None if t is None else t.to(DEV) for t in (q, k, pos, freq, wq, wk)]
    qo, ko = mb.rotate_qk(*dev, eps=eps, interleaved=inter, amplitude=amp)
    got = mb.rotate_qk_bwd(*dev[:4], gq.to(DEV), None if gk is None else gk.to(DEV), *dev[4:], eps=eps, interleaved=inter,
                           amplitude=amp)
    torch.cuda.synchronize()
    base = 0.0 if dtype == "f32" else 2.0 ** -8
    f = freq.numpy() if rot else np.zeros(0, np.float32)
    for name, x, w, g, y, dx, dw in (("q", q, wq, gq, qo, got[0], got[2]), ("k", k, wk, gk, ko, got[1], got[3])):
        if x is None:
            assert y is None and dx is None and dw is None
            continue
        assert y.dtype == dx.dtype == dt
        (r, m), (rx, mx), gw = ref.rotate(x.double().numpy(), None if w is None else w.numpy(), pos.numpy(), f, eps, amp,
                                          inter, g.double().numpy())
        e = cond_err(y.double().cpu().numpy(), r, m)
        assert e <= base + 2e-6, (name, e)
        e = cond_err(dx.double().cpu().numpy(), rx, mx)
        assert e <= base + 4e-6, ("d" + name, e)
        assert (dw is None) == (gw is None)
        if gw is not None:
            e = cond_err(dw.double().cpu().numpy(), *gw)
            assert e <= 8e-6, ("dw" + name, e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(8, 8), (8, 2), (16, 6), (64, 64), (64, 32), (80, 20), (80, 80), (96, 24), (128, 128),
                                   (128, 64), (128, 126), (120, 60), (64, 0)])
def test_widths(dtype, inter, d, rot):
    check(dtype, 2, 13, 3, 2, d, rot, inter, seed=d + rot)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T", [(1, 1), (64, 1), (1, 700), (3, 333)])
@pytest.mark.parametrize("H,Hk", [(1, 0), (1, 1), (16, 16), (5, 2), (32, 8)])
def test_steps_and_heads(dtype, B, T, H, Hk):
    check(dtype, B, T if H < 16 else min(T, 100), H, Hk, 64, 64, False, seed=B + T + H)


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("inter", [False, True])
def test_norms(norm, inter):
    check("bf16", 2, 50, 4, 2, 64, 32, inter, norm)


@pytest.mark.parametrize("far", [0, 1 << 17, (1 << 31) - 6000])
def test_far_positions(far):
    """The fraction of a turn is right to 2^-24 at any int32 position: the angle in
    64 bits has 2^31 2^-53 of a turn left, far below."""
    check("f32", 1, 64, 2, 2, 128, 128, False, (False, False), far=far)


def test_amplitude_and_eps():
    check("f32", 1, 40, 2, 1, 64, 32, False, amp=1.3, eps=0.5)
    check("f32", 1, 40, 3, 1, 80, 80, True, amp=-0.7, eps=0.0)


def test_rows_of_zeros_and_nonfinite_rows():
    announce("rotate zeros, nan, inf")
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    x = torch.randn(1, 3, 5, 64, device=DEV, generator=g)
    x[0, 0, 1] = 0
    x[0, 1, 2, 5] = float("nan")
    x[0, 2, 4, 60] = float("inf")
    w = torch.ones(64, device=DEV)
    pos = torch.arange(3, dtype=torch.int32, device=DEV)[None]
    y, _ = mb.rotate_qk(x, None, pos, mb.rotary_frequencies(64, device=DEV), w)
    assert not bool(y[0, 0, 1].any())
    bad = ~torch.isfinite(y).all(-1)
    assert bad.nonzero().tolist() == [[0, 1, 2], [0, 2, 4]]      # nothing leaves its row


def test_scaled_frequencies():
    f = mb.rotary_frequencies(64).double()
    assert torch.equal(mb.rotary_frequencies(64, factor=4.0).double(), (10000.0 ** (-torch.arange(0, 64, 2).double() / 64) / 4).float().double())
    y = mb.rotary_frequencies(64, factor=4.0, original_length=4096).double()
    turns = 4096 * f / (2 * np.pi)
    assert torch.equal(y[turns > 32.1], f[turns > 32.1])
    assert torch.allclose(y[turns < 0.99], f[turns < 0.99] / 4, rtol=1e-6)
    mid = (turns > 1.1) & (turns < 31)
    assert bool(((y < f) & (y > f / 4))[mid].all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_autograd_and_difference(dtype):
    announce("rotate autograd %s" % dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    dt = DT[dtype]
    q, k = (torch.randn(2, 9, h, 64, device=DEV, generator=g).to(dt).requires_grad_(True) for h in (4, 2))
    wq, wk = (torch.rand(64, device=DEV, generator=g).add(0.5).requires_grad_(True) for _ in range(2))
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    pos = torch.arange(9, dtype=torch.int32, device=DEV).expand(2, 9).contiguous()
    freq = mb.rotary_frequencies(32, device=DEV)
    out = mb.qk_rotate(q, k, pos, freq, wq, wk)
    torch.autograd.backward(out, (gq, gk))
    want = mb.rotate_qk_bwd(q.detach(), k.detach(), pos, freq, gq, gk, wq.detach(), wk.detach())
    for x, y in zip((q, k, wq, wk), want):
        assert torch.equal(x.grad, y)
    if dtype == "bf16":
        return
    # along a random direction: the fp32 forward (2e-6 of some 50 |L|^(1/2) terms)
    # over a step of 0.02 leaves 1e-2 of the derivative
    d = [torch.randn(x.shape, device=DEV, generator=g) for x in (q, k, wq, wk)]

    def loss(t):
        with torch.no_grad():
            x = [a + t * b for a, b in zip((q, k, wq, wk), d)]
            a, b = mb.rotate_qk(x[0], x[1], pos, freq, x[2], x[3])
        return float((a.double() * gq.double()).sum() + (b.double() * gk.double()).sum())

    num = (loss(0.01) - loss(-0.01)) / 0.02
    dot = sum(float((y.double() * b.double()).sum()) for y, b in zip(want, d))
    size = sum(float((y.double() * b.double()).square().sum()) for y, b in zip(want, d)) ** 0.5
    assert abs(num - dot) <= 1e-2 * max(abs(dot), size)


def test_graph_stream_and_workspace():
    announce("rotate graph")
    q, k = torch.randn(1, 300, 4, 64, device=DEV).bfloat16(), torch.randn(1, 300, 2, 64, device=DEV).bfloat16()
    w = torch.rand(64, device=DEV)
    pos = torch.arange(300, dtype=torch.int32, device=DEV)[None]
    freq = mb.rotary_frequencies(64, device=DEV)

    def both(ws=None):
        return mb.rotate_qk(q, k, pos, freq, w, w) + mb.rotate_qk_bwd(q, k, pos, freq, k.repeat(1, 1, 2, 1), k, w, w,
                                                                      workspace=ws)
    both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = both()
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(other, both()):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(3):
        q.copy_(torch.roll(q, 1, 1))
        k.copy_(torch.roll(k, 2, 1))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, both()):
            assert torch.equal(x, y)
    ws = torch.randint(0, 256, (mb.memoroid_rotate_qk_bwd_workspace_bytes(300, 4, 2, 64, 64, 0, mb.BF16),),
                       dtype=torch.uint8, device=DEV)
    for x, y in zip(both(ws), both()):
        assert torch.equal(x, y)
    assert mb.workspace_status(ws) == mb.OK


def test_rotated_retention_trains_as_its_formula():
    """The operators as a layer has them: norms and rotation, then retention, through
    autograd, against 64 bits; decode step by step gives the same."""
    import retention_ref as rr
    announce("rotate + retention")
    rng = np.random.default_rng(5)
    B, T, H, Hk, d = 2, 75, 4, 2, 64
    x = {n: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)) for n, s in
         (("q", (B, T, H, d)), ("k", (B, T, Hk, d)), ("v", (B, T, Hk, d)), ("g", (B, T, H, d)))}
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32))
    alpha = torch.tensor([0.3, 0.01, -0.05, 0.002])
    start = torch.from_numpy((rng.random((B, T)) < 0.05).astype(np.uint8))
    pos = torch.arange(T, dtype=torch.int32).expand(B, T).contiguous()
    freq = mb.rotary_frequencies(d)
    q, k, v, wd = (t.to(DEV).requires_grad_(True) for t in (x["q"], x["k"], x["v"], w))
    args = pos.to(DEV), freq.to(DEV)
    al, st = alpha.to(DEV), start.to(DEV)
    qr, kr = mb.qk_rotate(q, k, *args, wd, wd)
    out = mb.retention(qr, kr, v, al, st)
    out.backward(x["g"].to(DEV))
    # 64 bits
    f = freq.numpy()
    n64 = {n: t.double().numpy() for n, t in x.items()}
    r_q = ref.rotate(n64["q"], w.numpy(), pos.numpy(), f, 1e-6, 1.0, False)[0][0]
    r_k = ref.rotate(n64["k"], w.numpy(), pos.numpy(), f, 1e-6, 1.0, False)[0][0]
    sc = d ** -0.5
    want = rr.forward(r_q, r_k, n64["v"], alpha.numpy(), start.numpy(), sc)[0]
    b = rr.backward(r_q, r_k, n64["v"], alpha.numpy(), start.numpy(), sc, n64["g"])
    dq = ref.rotate(n64["q"], w.numpy(), pos.numpy(), f, 1e-6, 1.0, False, b["dq"])
    dk = ref.rotate(n64["k"], w.numpy(), pos.numpy(), f, 1e-6, 1.0, False, b["dk"])
    # each step's 4e-6 / 2e-5 of magnitudes that are up to some 20 times the values
    for got, r in ((out.detach(), want), (q.grad, dq[1][0]), (k.grad, dk[1][0]), (v.grad, b["dv"]),
                   (wd.grad, dq[2][0] + dk[2][0])):
        got = got.double().cpu().numpy()
        assert np.abs(got - r).max() <= 20 * 2.4e-5 * np.abs(r).max()
    S = torch.zeros(B, H, d, d, device=DEV)
    for t in range(T):
        with torch.no_grad():
            a, c = mb.rotate_qk(q[:, t].contiguous(), k[:, t].contiguous(), args[0][:, t].contiguous(), args[1], wd, wd)
            o = mb.retention_step(a, c, v[:, t].contiguous(), al, S, st[:, t].contiguous())
        assert np.abs(o.double().cpu().numpy() - want[:, t]).max() <= 20 * 2.4e-5 * np.abs(want).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_alone(dtype):
    """No query heads: q and its gradients may be missing, and their weight's
    gradient is zero."""
    n, Hk, d = 37, 3, 64
    announce("rotate H=0 %s" % dtype)
    dt = DT[dtype]
    code = mb.F32 if dtype == "f32" else mb.BF16
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    k, gk = (torch.randn(n, Hk, d, generator=g, device=DEV).to(dt) for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    freq = mb.rotary_frequencies(d, device=DEV)
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    want, _ = mb.rotate_qk(k, None, pos, freq, w)
    want_k, _, want_w, _ = mb.rotate_qk_bwd(k, None, pos, freq, gk, None, w)
    out, dk = torch.empty_like(k), torch.empty_like(k)
    dwq, dwk = torch.full_like(w, 7.0), torch.full_like(w, 7.0)
    s = torch.cuda.current_stream().cuda_stream
    assert mb.memoroid_rotate_qk(None, k.data_ptr(), pos.data_ptr(), freq.data_ptr(), w.data_ptr(), w.data_ptr(), None,
                                 out.data_ptr(), 1e-6, 1.0, 0, n, 0, Hk, d, d, code, s) == mb.OK
    nb = mb.memoroid_rotate_qk_bwd_workspace_bytes(n, 0, Hk, d, d, 0, code)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    assert mb.memoroid_rotate_qk_bwd(None, k.data_ptr(), pos.data_ptr(), freq.data_ptr(), w.data_ptr(), w.data_ptr(), None,
                                     gk.data_ptr(), None, dk.data_ptr(), dwq.data_ptr(), dwk.data_ptr(), 1e-6, 1.0, 0, n, 0,
                                     Hk, d, d, code, ws.data_ptr(), nb, s) == mb.OK
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(dk, want_k) and torch.equal(dwk, want_w)
    assert not bool(dwq.any())


def test_more_than_2_31_elements():
    """Rows past 2^31 elements are the rows of a call of their own."""
    n, H, d, tail = 560000, 32, 128, 50
    announce("rotate n=%d H=%d d=%d bf16" % (n, H, d))
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    q, gq = (torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    assert q.numel() > 1 << 31
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    freq = mb.rotary_frequencies(d, device=DEV)
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    out = mb.rotate_qk(q, None, pos, freq, w)[0]
    dq = mb.rotate_qk_bwd(q, None, pos, freq, gq, None, w)[0]
    for rows in (slice(0, tail), slice(n - tail, n)):
        x, gx, p = q[rows].contiguous(), gq[rows].contiguous(), pos[rows].contiguous()
        assert torch.equal(out[rows], mb.rotate_qk(x, None, p, freq, w)[0])
        assert torch.equal(dq[rows], mb.rotate_qk_bwd(x, None, p, freq, gx, None, w)[0])


def test_two_graphs_of_training_steps():
    """Forward and backward through autograd captured twice, replayed in turn with
    eager calls between."""
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    B, T, H, Hk, d = 2, 150, 4, 2, 64
    freq = mb.rotary_frequencies(d, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV).repeat(B, 1)
    sets = [[torch.randn(B, T, h, d, generator=g, device=DEV) for h in (H, Hk, H, Hk)] +
            [1 + 0.2 * torch.randn(d, generator=g, device=DEV) for _ in range(2)] for _ in range(2)]

    def step(q, k, gq, gk, wq, wk):
        x = [t.detach().requires_grad_(True) for t in (q, k, wq, wk)]
        out = mb.qk_rotate(x[0], x[1], pos, freq, x[2], x[3])
        return out + torch.autograd.grad(out, x, (gq, gk))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c in sets:
            step(*c)
    torch.cuda.current_stream().wait_stream(s)
    graphs, results = [], []
    for c in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            results.append([y.detach() for y in step(*c)])
    for i in range(4):
        for c in sets:
            for t in c[:4]:
                t.copy_(torch.roll(t, 1 + i, 1))
        for j in (0, 1) if i % 2 else (1, 0):
            graphs[j].replay()
        torch.cuda.synchronize()
        for c, y in zip(sets, results):
            for a, b in zip(step(*c), y):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,value", [("f32", 0.1), ("bf16", 0.7)])
@pytest.mark.parametrize("rows", [4096, 40960])
def test_weight_gradient_of_many_rows(dtype, value, rows):
    """One key head beside 2047 query heads has few lanes, each with `rows` of its rows:
    sums of equal terms, whose roundings in floats all go one way, against the product.
    No sum of floats is longer than 64 of them, so the bound above holds: 8e-6."""
    announce("rotate weights' gradient, %s, %d rows a lane" % (dtype, rows))
    n, H, d = 4 * rows, 2047, 8                             # four wavefronts for the key head
    q = torch.ones(n, H, d, dtype=DT[dtype], device=DEV)
    k = torch.ones(n, 1, d, dtype=DT[dtype], device=DEV)
    gk = torch.full_like(k, value)
    w = torch.ones(d, device=DEV)
    got = mb.rotate_qk_bwd(q, k, None, None, q, gk, w, w)
    for dw, g, heads in ((got[2], 1.0, H), (got[3], float(gk[0, 0, 0].double()), 1)):
        want = n * heads * g / np.sqrt(1.0 + float(np.float32(1e-6)))
        e = float((dw.double() / want - 1).abs().max())
        print("  %.1e" % e, flush=True)
        assert e <= 8e-6


def test_weight_gradient_past_2_31_elements():
    """Against blocked 64-bit sums, relative to the sum over absolute values."""
    n, H, d = 560000, 32, 128
    announce("rotate weights' gradient n=%d H=%d d=%d bf16" % (n, H, d))
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    q, gq = (torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    assert q.numel() > 1 << 31
    gq.abs_()
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    dw = mb.rotate_qk_bwd(q, None, None, None, gq, None, w)[2]
    want, size = (torch.zeros(d, dtype=torch.float64, device=DEV) for _ in range(2))
    for i in range(0, n, 20000):
        x = q[i:i + 20000].double()
        t = gq[i:i + 20000].double() * x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        want += t.sum((0, 1))
        size += t.abs().sum((0, 1))
    e = float(((dw.double() - want).abs() / size).max())
    print("  %.1e" % e, flush=True)
    assert e <= 8e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 32), (80, 20), (16, 6), (8, 2), (64, 0)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_nonfinite_values_behind_the_turned_part(dtype, inter, d, rot, value):
    """Elements rot .. d - 1 stay as they are, an infinity or NaN among them too, and
    change no other element: without a norm every row is that of finite values, apart
    from the element itself; in both directions."""
    announce("rotate nonfinite %s inter=%d d=%d rot=%d" % (dtype, inter, d, rot))
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    x = torch.randn(d - rot, 3, d, generator=g, device=DEV).to(DT[dtype])
    bad = x.clone()
    i = torch.arange(d - rot, device=DEV)
    bad[i, 1, rot + i] = value                              # each of them in a step of its own
    pos = torch.arange(d - rot, dtype=torch.int32, device=DEV)
    freq = mb.rotary_frequencies(rot, device=DEV) if rot else None
    for call in (lambda t: mb.rotate_qk(t, None, pos, freq, interleaved=inter, amplitude=1.5)[0],
                 lambda t: mb.rotate_qk_bwd(t, None, pos, freq, t, None, interleaved=inter, amplitude=1.5)[0]):
        want = call(x)
        assert torch.equal(want[..., rot:], x[..., rot:])
        want[i, 1, rot + i] = value
        assert torch.equal(torch.nan_to_num(call(bad), nan=-1e6), torch.nan_to_num(want, nan=-1e6))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_heads(dtype):
    check(dtype, 1, 3, 65535, 65535, 8, 8, False, seed=1)
