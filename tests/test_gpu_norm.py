"""Layer norm and dropout on the GPU against gated_ref.py, errors relative to max(|r|, m).

Tolerances, in E = 2^-24 (half a step of fp32, relative), for rows of d elements.  A row's
sum of d fp32 values goes through at most ceil(d / 64) / 8 octets a lane, eight adds each,
and 10 steps across lanes and wavefronts; 16384 columns in 1024 lanes are 16 adds and 10, 2048 in
64 lanes 32 and 6: below 40 E of the sum of magnitudes, as are the sum of squares, relative to
itself; mean, deviation, root, reciprocal and the products add ten.  y: the mean's
error counts with the row's mean magnitude (in m), rstd's 25 E with y's: 80 E.  ds
goes through xh twice and two more sums: 240 E.  dw and db add the rows of a lane, at
most 64 of them, then at most 64 wavefronts' in doubles: 80 + 64 E.  dropout and the sum with the
residual: 3 E.  bf16: the rounding of the result, 2^-8, and the same."""
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
SEED, STEP, SITE = 0x1234567890ABCDEF, (7 << 32) + 99, 5


def base(dtype):
    return 0.0 if dtype == "f32" else 2.0 ** -8


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def rng_tensor(seed=SEED, step=STEP):
    return torch.tensor([seed, step], dtype=torch.int64, device=DEV)


def inputs(dtype, shape, residual, weights, seed):
    rng = np.random.default_rng(seed)
    dt = DT[dtype]

    def normal(*sh):
        return torch.from_numpy(rng.standard_normal(sh, dtype=np.float32))

    d = shape[-1]
    s = dict(x=normal(*shape).to(dt), gy=normal(*shape).to(dt))
    s["res"] = (normal(*shape) * torch.exp(0.5 * normal(d)) + normal(d)).to(dt) if residual else None
    s["gs"] = normal(*shape).to(dt) if residual else None
    s["w"], s["b"] = (1 + 0.2 * normal(d), 0.3 * normal(d)) if weights else (None, None)
    return s


def summed(s, p, mask):
    x = np64(s["x"])
    t = np.where(mask, x / (1 - p), 0.0) if mask is not None else x
    m = np.abs(t)
    return (t, m) if s["res"] is None else (t + np64(s["res"]), m + np.abs(np64(s["res"])))


def check(dtype, shape, residual=True, p=0.0, weights=True, eps=1e-5, seed=0):
    announce("norm %s %s residual=%s p=%g weights=%s" % (dtype, shape, residual, p, weights))
    s = inputs(dtype, shape, residual, weights, seed)
    c = {k: None if v is None else v.to(DEV) for k, v in s.items()}
    rng = rng_tensor() if p else None
    got = mb.norm_rows(c["x"], c["w"], c["b"], eps, c["res"], p, rng, SITE, keep_stats=True)
    y, stats = got[0], got[-1]
    dx, dres, dw, db = mb.norm_rows_bwd(c["x"], stats, c["gy"], c["w"], c["res"], c["gs"], p, rng, SITE)
    torch.cuda.synchronize()
    n, d = int(np.prod(shape[:-1])), shape[-1]
    mask = ref.keep(p, SEED, STEP, SITE, n, d).reshape(shape) if p else None
    t, mt = summed(s, p, mask)
    w, b = (None if v is None else v.numpy() for v in (s["w"], s["b"]))
    ry, my, mean, r = ref.norm(t, w, b, eps, mt)
    assert cond_err(np64(y), ry, my) <= base(dtype) + 80 * E
    if residual or p:
        assert len(got) == 3
        assert cond_err(np64(got[1]), t, mt) <= base(dtype) + 3 * E
    else:
        assert len(got) == 2
    assert cond_err(np64(stats[..., :1]), mean, mt.mean(-1, keepdims=True)) <= 45 * E
    (ds, ms), gw, gb = ref.norm_grads(t, w, eps, np64(s["gy"]), np64(s["gs"]))
    if residual:
        assert (dres.data_ptr() == dx.data_ptr()) == (p == 0)
        assert cond_err(np64(dres), ds, ms) <= base(dtype) + 240 * E
    else:
        assert dres is None
    on = 1.0 if mask is None else mask / (1 - p)
    assert cond_err(np64(dx), ds * on, ms * on) <= base(dtype) + 243 * E
    if mask is not None:
        assert not bool(dx.cpu().numpy(force=True)[~mask].any() if dtype == "f32" else dx.float().cpu().numpy()[~mask].any())
    assert cond_err(np64(dw), *gw) <= 144 * E
    assert cond_err(np64(db), *gb) <= 144 * E
    assert dw.dtype == db.dtype == stats.dtype == torch.float32 and y.dtype == dx.dtype == DT[dtype]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 2, 7, 8, 9, 31, 50, 64, 250, 256, 512, 513, 1000, 1024, 1031, 2048])
def test_widths(dtype, d):
    check(dtype, (3, 11, d), seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [2049, 4096, 4099, 8192, 8200, 16383, 16384])
def test_wide_rows(dtype, d):
    check(dtype, (5, d), seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 256), (2, 1, 64), (257, 40), (4097, 64), (70000, 8), (3000, 1), (9000, 256), (2500, 2048),
                                   (64,)])
def test_rows(dtype, shape):
    check(dtype, shape, seed=len(shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("weights", [False, True])
def test_variants(dtype, residual, p, weights):
    check(dtype, (37, 70), residual, p, weights, eps=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 64, 600, 1500, 3000, 5000, 9000])
def test_dropout_in_the_norm(dtype, d):
    check(dtype, (9, d), True, 0.25, seed=d)


def test_offset_rows():
    """A mean 100 times the deviation: the deviation is taken before the squares."""
    announce("norm offset")
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((20, 512)) + 100).astype(np.float32)
    y = mb.norm_rows(torch.from_numpy(x).to(DEV))
    ry, my, _, _ = ref.norm(x, None, None, 1e-5)
    assert cond_err(np64(y), ry, my) <= 80 * E


def test_equal_and_bad_rows():
    announce("norm equal, nan and inf rows")
    x = torch.randn(6, 96, device=DEV)
    x[1] = 3.0
    x[2, 5] = float("nan")
    x[4, 95] = float("inf")
    w, b = torch.rand(96, device=DEV), torch.randn(96, device=DEV)
    y, st = mb.norm_rows(x, w, b, keep_stats=True)
    assert torch.equal(y[1], b)
    assert (~torch.isfinite(y).all(-1)).nonzero().flatten().tolist() == [2, 4]
    dx, _, _, _ = mb.norm_rows_bwd(x, st, torch.randn_like(x), w)
    assert (~torch.isfinite(dx).all(-1)).nonzero().flatten().tolist() == [2, 4]


def test_all_dropped():
    """p = 1: the norm is that of the residual, x takes part in nothing and gets no gradient."""
    announce("norm p=1")
    for d in (64, 1500):
        x = torch.full((9, d), float("nan"), device=DEV, requires_grad=True)
        res, w = torch.randn(9, d, device=DEV).requires_grad_(True), torch.rand(d, device=DEV)
        gy, gs = torch.randn(9, d, device=DEV), torch.randn(9, d, device=DEV)
        y, s = mb.layer_norm(x, w, residual=res, p=1.0, rng=rng_tensor())
        dx, dres = torch.autograd.grad((y, s), (x, res), (gy, gs))
        assert torch.equal(s, res) and not bool(dx.any()) and torch.equal(y, mb.norm_rows(res.detach(), w))
        zero = torch.zeros(9, d, device=DEV).requires_grad_(True)
        y, s = mb.layer_norm(zero, w, residual=res, p=0.0)
        assert torch.equal(dres, torch.autograd.grad((y, s), res, (gy, gs))[0])


def test_overflow():
    """Rows whose squared deviations are past fp32's range come out as the bias; large ones
    below that do not."""
    announce("norm overflow")
    b = torch.randn(256, device=DEV)
    z = torch.randn(4, 256, device=DEV)
    y = mb.norm_rows(z * 2.0 ** 66, None, b)
    assert torch.equal(y, b.expand_as(y))
    assert torch.equal(mb.norm_rows(z * 2.0 ** 56, eps=0.0), mb.norm_rows(z, eps=0.0))


def test_no_rows_and_no_columns():
    announce("norm empty")
    w = torch.ones(8, device=DEV)
    y, st = mb.norm_rows(torch.zeros(0, 8, device=DEV), w, keep_stats=True)
    dx, dr, dw, db = mb.norm_rows_bwd(torch.zeros(0, 8, device=DEV), st, torch.zeros(0, 8, device=DEV), w)
    assert y.shape == dx.shape == (0, 8) and dr is None and not bool(dw.any()) and not bool(db.any())
    assert mb.norm_rows(torch.zeros(4, 0, device=DEV)).shape == (4, 0)
    assert mb.drop_rows(torch.zeros(0, 8, device=DEV), 0.5, rng_tensor()).shape == (0, 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_autograd(dtype):
    announce("norm autograd %s" % dtype)
    s = inputs(dtype, (4, 30, 72), True, True, 3)
    c = {k: v.to(DEV) for k, v in s.items()}
    rng = rng_tensor()
    leaves = [c[k].clone().requires_grad_(True) for k in ("x", "w", "b", "res")]
    y, t = mb.layer_norm(*leaves[:3], residual=leaves[3], p=0.2, rng=rng, site=SITE)
    torch.autograd.backward((y, t), (c["gy"], c["gs"]))
    _, _, st = mb.norm_rows(c["x"], c["w"], c["b"], residual=c["res"], p=0.2, rng=rng, site=SITE, keep_stats=True)
    want = mb.norm_rows_bwd(c["x"], st, c["gy"], c["w"], c["res"], c["gs"], 0.2, rng, SITE)
    for x, g in zip((leaves[0], leaves[3], leaves[1], leaves[2]), want):
        assert torch.equal(x.grad, g)
    # one output alone; gradients that are views; no weights
    y, t = mb.layer_norm(leaves[0], residual=leaves[3])
    gx, gr = torch.autograd.grad(t.float().sum(), (leaves[0], leaves[3]))
    assert torch.equal(gx, torch.ones_like(gx)) and torch.equal(gr, torch.ones_like(gr))
    y = mb.layer_norm(leaves[0], leaves[1])
    gw, = torch.autograd.grad(y, leaves[1:2], c["gy"])
    _, st = mb.norm_rows(c["x"], c["w"], keep_stats=True)
    assert torch.equal(gw, mb.norm_rows_bwd(c["x"], st, c["gy"], c["w"])[2])
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(mb.layer_norm(*leaves[:3]).float().sum(), leaves[:1], create_graph=True)
        g.float().sum().backward()


def test_one_leaf_as_x_and_residual():
    announce("norm one leaf twice")
    x = torch.randn(5, 40, device=DEV, requires_grad=True)
    y, s = mb.layer_norm(x, residual=x)
    g = torch.randn_like(y)
    gx, = torch.autograd.grad((y, s), x, (g, g))
    _, _, st = mb.norm_rows(x.detach(), residual=x.detach(), keep_stats=True)
    want = mb.norm_rows_bwd(x.detach(), st, g, residual=x.detach(), grad_s=g)[0]
    assert torch.equal(gx, 2 * want)


def test_norm_differences():
    announce("norm differences")
    s = inputs("f32", (6, 50), True, True, 8)
    c = {k: v.to(DEV) for k, v in s.items()}
    rng = rng_tensor()
    names = ("x", "w", "b", "res")
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    v = {k: torch.randn(c[k].shape, generator=g, device=DEV) for k in names}

    def value(t):
        a = {k: c[k] + t * v[k] for k in names}
        y, u = mb.norm_rows(a["x"], a["w"], a["b"], 1e-5, a["res"], 0.3, rng, SITE)
        return float((y.double() * c["gy"].double()).sum() + (u.double() * c["gs"].double()).sum())

    eps = 2.0 ** -7
    want = (8 * (value(eps) - value(-eps)) - (value(2 * eps) - value(-2 * eps))) / (12 * eps)
    _, _, st = mb.norm_rows(c["x"], c["w"], c["b"], 1e-5, c["res"], 0.3, rng, SITE, keep_stats=True)
    dx, dr, dw, db = mb.norm_rows_bwd(c["x"], st, c["gy"], c["w"], c["res"], c["gs"], 0.3, rng, SITE)
    terms = [float((y.double() * v[k].double()).sum()) for k, y in zip(("x", "res", "w", "b"), (dx, dr, dw, db))]
    assert abs(sum(terms) - want) <= 1e-3 * sum(abs(t) for t in terms), (terms, want)


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (5, 3), (3, 8), (7, 9), (2, 3, 250), (100, 64), (1, 4099), (4099,), (33, 1000)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.97])
def test_dropout(dtype, shape, p):
    announce("dropout %s %s p=%g" % (dtype, shape, p))
    s = inputs(dtype, shape, True, False, 1)
    c = {k: None if v is None else v.to(DEV) for k, v in s.items()}
    rng = rng_tensor()
    n, d = int(np.prod(shape[:-1], dtype=np.int64)), shape[-1]
    mask = ref.keep(p, SEED, STEP, SITE, n, d).reshape(shape)
    for res in (None, s["res"]):
        out = mb.drop_rows(c["x"], p, rng, SITE, None if res is None else c["res"])
        t, mt = summed(dict(x=s["x"], res=res), p, mask)
        assert cond_err(np64(out), t, mt) <= base(dtype) + 3 * E
        if res is None:
            assert bool((out.cpu().numpy(force=True) == 0)[~mask].all() if dtype == "f32" else
                        (out.float().cpu().numpy() == 0)[~mask].all())
    # through autograd: the same mask on the gradient
    x, r = (c[k].clone().requires_grad_(True) for k in ("x", "res"))
    gx, gr = torch.autograd.grad(mb.dropout(x, p, rng, SITE, r), (x, r), c["gy"])
    assert torch.equal(gr, c["gy"])
    assert torch.equal(gx, mb.drop_rows(c["gy"], p, rng, SITE))


def test_limits_of_p():
    """p = 1 drops all, NaN and Inf too; a p whose limit has lower halves at work: elements
    whose upper half ties with it are settled by the lower one."""
    announce("dropout limits")
    x = torch.full((4, 100), float("nan"), device=DEV)
    r = torch.randn(4, 100, device=DEV)
    assert torch.equal(mb.drop_rows(x, 1.0, rng_tensor(), 0, r), r)
    assert not bool(mb.drop_rows(x, 1.0, rng_tensor()).any())
    rows, d = 16, 4096
    u = ref.numbers(SEED, STEP, SITE, rows, d)
    # limits right at and right above an element's own number, and around its upper half
    for i, j in ((0, 0), (3, 77), (15, 4095)):
        v = int(u[i, j])
        for limit in (v, v + 1, v & ~0xFFFF, (v | 0xFFFF) + 1):
            if not 0 < limit <= 1 << 32:
                continue
            out = mb.drop_rows(torch.ones(rows, d, device=DEV), limit * 2.0 ** -32, rng_tensor(), SITE)
            assert np.array_equal(out.cpu().numpy() != 0, u >= np.uint64(limit)), (i, j, limit)


def test_numbers_depend_on_all_their_inputs():
    announce("dropout inputs")
    x = torch.ones(64, 64, device=DEV)
    first = mb.drop_rows(x, 0.5, rng_tensor(), 0)
    assert torch.equal(first, mb.drop_rows(x, 0.5, rng_tensor(), 0))
    for rng, site in ((rng_tensor(SEED + 1), 0), (rng_tensor(SEED + (1 << 40)), 0), (rng_tensor(SEED, STEP + 1), 0),
                      (rng_tensor(), 1), (rng_tensor(), (1 << 32) - 1)):
        same = float((mb.drop_rows(x, 0.5, rng, site) == first).float().mean())
        assert abs(same - 0.5) < 0.05                      # 4096 elements: 6.4 standard deviations
    # the low 32 bits of the step count; negative seeds are numbers like any other
    assert torch.equal(first, mb.drop_rows(x, 0.5, rng_tensor(SEED, STEP + (1 << 32)), 0))
    assert bool(mb.drop_rows(x, 0.5, rng_tensor(-1), 0).any())


def test_share_that_stays():
    """2^22 elements at p = 0.1: the share is within 6 standard deviations, and so is
    every column's and every row's own."""
    announce("dropout share")
    n = 2048
    on = (mb.drop_rows(torch.ones(n, n, device=DEV), 0.1, rng_tensor(), 2) != 0).double()
    assert abs(float(on.mean()) - 0.9) < 6 * 0.3 / n
    for m in (on.mean(0), on.mean(1)):
        assert float((m - 0.9).abs().max()) < 6 * 0.3 / n ** 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_changed_rng_is_refused(dtype):
    announce("dropout changed rng")
    rng = rng_tensor()
    x = torch.randn(4, 16, device=DEV).to(DT[dtype]).requires_grad_(True)
    out = mb.dropout(x, 0.5, rng)
    y, _ = mb.layer_norm(x, p=0.5, rng=rng)
    rng[1] += 1
    for t in (out, y):
        with pytest.raises(RuntimeError):
            t.float().sum().backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [37, 64, 1500, 5001])
def test_odd_addresses_and_nothing_behind(dtype, d):
    """Operands that start one element into their memory, outputs with guards around."""
    announce("norm guards %s d=%d" % (dtype, d))
    n = 7
    s = inputs(dtype, (n, d), True, True, 2)
    rng = rng_tensor()
    c = {k: v.to(DEV) for k, v in s.items()}
    want = mb.norm_rows(c["x"], c["w"], c["b"], 1e-5, c["res"], 0.2, rng, SITE, keep_stats=True)
    want += mb.norm_rows_bwd(c["x"], want[2], c["gy"], c["w"], c["res"], c["gs"], 0.2, rng, SITE)
    want += (mb.drop_rows(c["x"], 0.2, rng, SITE, c["res"]),)

    def shifted(t):
        buf = torch.full((t.numel() + 130,), 7, dtype=t.dtype, device=DEV)
        view = buf[65:65 + t.numel()].view(t.shape)
        view.copy_(t)
        return buf, view

    i = {k: shifted(v)[1] for k, v in s.items()}
    p = {k: v.data_ptr() for k, v in i.items()}
    outs = [shifted(torch.zeros_like(t)) for t in want]
    o = [v.data_ptr() for _, v in outs]
    dt = mb.F32 if dtype == "f32" else mb.BF16
    need = mb.memoroid_layer_norm_bwd_workspace_bytes(n, d)
    ws = torch.randint(0, 256, (need + 512,), dtype=torch.uint8, device=DEV)
    keep = ws[need:].clone()
    st = torch.cuda.current_stream().cuda_stream
    assert mb.memoroid_layer_norm(p["x"], p["res"], p["w"], p["b"], rng.data_ptr(), o[0], o[1], o[2], 1e-5, 0.2, SITE, n, d, dt,
                                  st) == mb.OK
    assert mb.memoroid_layer_norm_bwd(p["x"], p["res"], p["w"], rng.data_ptr(), o[2], p["gy"], p["gs"], o[3], o[4], o[5], o[6],
                                      0.2, SITE, n, d, dt, ws.data_ptr(), need, st) == mb.OK
    assert mb.memoroid_dropout(p["x"], p["res"], rng.data_ptr(), o[7], 0.2, SITE, n, d, dt, st) == mb.OK
    torch.cuda.synchronize()
    for (buf, view), w in zip(outs, want):
        assert torch.equal(view, w)
        assert bool((buf[:65] == 7).all()) and bool((buf[65 + w.numel():] == 7).all())
    assert torch.equal(ws[need:], keep)


def test_past_32_bits():
    """More than 2^31 elements: the last rows are what they are alone (dropout's numbers
    go by the row, so those rows are compared without it)."""
    announce("norm past 2^31 elements")
    n, d, m = 1050000, 2048, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.zeros(n, d, dtype=torch.bfloat16, device=DEV)
    x[-m:] = torch.randn(m, d, device=DEV, generator=g).to(torch.bfloat16)
    w, b = torch.rand(d, device=DEV, generator=g), torch.randn(d, device=DEV, generator=g)
    y, s, st = mb.norm_rows(x, w, b, residual=x, keep_stats=True)
    yl, sl, stl = mb.norm_rows(x[-m:], w, b, residual=x[-m:], keep_stats=True)
    assert torch.equal(y[-m:], yl) and torch.equal(s[-m:], sl) and torch.equal(st[-m:], stl)
    assert torch.equal(y[0], b.to(torch.bfloat16))
    dx, _, dw, db = mb.norm_rows_bwd(x, st, x, w)
    dxl, _, dwl, dbl = mb.norm_rows_bwd(x[-m:], stl, x[-m:], w)
    assert torch.equal(dx[-m:], dxl)
    assert float((db - dbl).abs().max()) <= 144 * E * float(x[-m:].abs().double().sum(0).max())
    del y, s, dx
    out = mb.drop_rows(x, 0.5, rng_tensor(), SITE, x)
    mask = ref.keep(0.5, SEED, STEP, SITE, 2, d, first_row=n - 2)
    assert np.array_equal(np64(out[-2:]), np64((x[-2:].double() * torch.from_numpy(1.0 + 2.0 * mask).to(DEV)).to(torch.bfloat16)))


def test_runs_are_equal():
    announce("norm equal runs")
    s = inputs("bf16", (5000, 192), True, True, 4)
    c = {k: v.to(DEV) for k, v in s.items()}
    rng = rng_tensor()
    first = None
    for _ in range(4):
        got = mb.norm_rows(c["x"], c["w"], c["b"], 1e-5, c["res"], 0.1, rng, SITE, keep_stats=True)
        got += mb.norm_rows_bwd(c["x"], got[2], c["gy"], c["w"], c["res"], c["gs"], 0.1, rng, SITE)
        if first is None:
            first = [t.clone() for t in got]
        assert all(torch.equal(x, y) for x, y in zip(first, got))
