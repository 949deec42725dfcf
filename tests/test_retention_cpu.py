"""Retention on the CPU: the 64-bit reference against differences, the C entry
points' refusals (before any HIP call, on pointers that are never followed) and
the torch layer's."""
import numpy as np
import pytest

import retention_ref as ref
from paper_2402_09900_amd import binding as mb

torch = pytest.importorskip("torch")

P = [0x10000 * (i + 1) for i in range(16)]      # distinct, aligned, never followed


@pytest.mark.parametrize("carry", [False, True])
def test_reference_gradient_against_differences(carry):
    rng = np.random.default_rng(0)
    B, T, H, Hk, dk, dv = 2, 9, 4, 2, 3, 5
    x = dict(q=rng.standard_normal((B, T, H, dk)), k=rng.standard_normal((B, T, Hk, dk)),
             v=rng.standard_normal((B, T, Hk, dv)), alpha=rng.uniform(-0.5, 0.5, H),
             state=rng.standard_normal((B, H, dk, dv)) if carry else None)
    start = (rng.random((B, T)) < 0.2).astype(np.uint8)
    g = rng.standard_normal((B, T, H, dv))
    G = rng.standard_normal((B, H, dk, dv)) if carry else np.zeros((B, H, dk, dv))

    def loss(x):
        out, S, _ = ref.forward(x["q"], x["k"], x["v"], x["alpha"], start, 0.7, x["state"])
        return (out * g).sum() + (S * G).sum()

    b = ref.backward(x["q"], x["k"], x["v"], x["alpha"], start, 0.7, g, x["state"], G)
    for n in x:
        if x[n] is None:
            continue
        d, h = rng.standard_normal(x[n].shape), 1e-5
        num = (loss({**x, n: x[n] + h * d}) - loss({**x, n: x[n] - h * d})) / (2 * h)
        assert abs(num - (b["d" + n] * d).sum()) <= 1e-6 * (1 + abs(num)), n


def scan(q=P[0], k=P[1], v=P[2], alpha=P[3], start=P[4], state_in=P[5], out=P[6], state_out=P[7], scale=1.0, B=2, T=100,
         H=4, Hk=2, dk=64, dv=64, dtype=mb.F32, ws=P[8], nbytes=1 << 40):
    return mb.memoroid_scan_retention(q, k, v, alpha, start, state_in, out, state_out, scale, B, T, H, Hk, dk, dv, dtype,
                                      ws, nbytes, None)


def bwd(q=P[0], k=P[1], v=P[2], alpha=P[3], start=P[4], state_in=P[5], g=P[6], G=P[7], dq=P[8], dk_=P[9], dv_=P[10],
        da=P[11], ds=P[12], scale=1.0, B=2, T=100, H=4, Hk=2, dk=64, dv=64, dtype=mb.F32, ws=P[13], nbytes=1 << 40):
    return mb.memoroid_scan_retention_bwd(q, k, v, alpha, start, state_in, g, G, dq, dk_, dv_, da, ds, scale, B, T, H, Hk,
                                          dk, dv, dtype, ws, nbytes, None)


def step(q=P[0], k=P[1], v=P[2], alpha=P[3], start=P[4], state=P[5], out=P[6], scale=1.0, B=2, H=4, Hk=2, dk=64, dv=64,
         dtype=mb.F32):
    return mb.memoroid_retention_step(q, k, v, alpha, start, state, out, scale, B, H, Hk, dk, dv, dtype, None)


SIZES = [(dict(B=-1), mb.EINVAL), (dict(H=-4), mb.EINVAL), (dict(Hk=-1), mb.EINVAL), (dict(dk=-64), mb.EINVAL),
         (dict(Hk=0), mb.EINVAL), (dict(Hk=3), mb.EINVAL), (dict(H=2, Hk=4), mb.EINVAL),
         (dict(scale=float("nan")), mb.EINVAL), (dict(scale=float("inf")), mb.EINVAL),
         (dict(dk=60), mb.EUNSUPPORTED), (dict(dv=136), mb.EUNSUPPORTED), (dict(dk=0), mb.EUNSUPPORTED),
         (dict(dtype=mb.C64), mb.EUNSUPPORTED), (dict(dtype=7), mb.EUNSUPPORTED),
         (dict(H=65536, Hk=65536), mb.EUNSUPPORTED), (dict(B=0), mb.OK), (dict(H=0, Hk=0), mb.OK)]


@pytest.mark.parametrize("call", [scan, bwd, step])
@pytest.mark.parametrize("change,status", SIZES)
def test_sizes(call, change, status):
    assert call(**change) == status


@pytest.mark.parametrize("call", [scan, bwd])
def test_long_and_empty_tapes(call):
    assert call(T=0) == mb.OK
    assert call(T=-1) == mb.EINVAL
    assert call(T=1 << 31) == mb.EUNSUPPORTED
    assert call(B=65536) == mb.EUNSUPPORTED


def test_step_batch_limit():
    assert step(B=1 << 40) == mb.EUNSUPPORTED
    assert step(B=1 << 62) == mb.EUNSUPPORTED


def test_missing_pointers():
    for call, names in ((scan, "q k v alpha start out"), (bwd, "q k v alpha start g dq dk_ dv_"),
                        (step, "q k v alpha state out")):
        for n in names.split():
            assert call(**{n: None}) == mb.EINVAL, (call.__name__, n)


def test_alignment():
    for call, names in ((scan, "q k v state_in out state_out ws"), (bwd, "q k v state_in g G dq dk_ dv_ ds ws"),
                        (step, "q k v state out")):
        for n in names.split():
            assert call(**{n: 0x900008}) == mb.EINVAL, (call.__name__, n)
    for call in (scan, bwd, step):
        assert call(alpha=0x900002) == mb.EINVAL
    assert bwd(da=0x900002) == mb.EINVAL


def test_aliasing():
    for call, ins, outs in ((scan, "q k v alpha start state_in", "out state_out"),
                            (bwd, "q k v alpha start state_in g G", "dq dk_ dv_ da ds"),
                            (step, "q k v alpha start", "out state")):
        for o in outs.split():
            for i in ins.split():
                assert call(**{o: 0x900000, i: 0x900000}) == mb.EINVAL, (call.__name__, i, o)
            for o2 in outs.split():
                if o2 != o:
                    assert call(**{o: 0x900000, o2: 0x900000}) == mb.EINVAL, (call.__name__, o, o2)


def test_workspace_sizes():
    for dt in (mb.F32, mb.BF16):
        n = mb.memoroid_scan_retention_workspace_bytes(2, 5000, 4, 64, 96, dt)
        assert n >= 256
        assert scan(T=5000, dv=96, dtype=dt, nbytes=n - 1) == mb.EWORKSPACE
        assert scan(T=5000, dv=96, dtype=dt, ws=None) == mb.EWORKSPACE
        assert n <= mb.memoroid_workspace_bytes(mb.OP_RETENTION, 2, 5000, 4, 64, 96, 0)
        for alpha in (0, 1):
            n = mb.memoroid_scan_retention_bwd_workspace_bytes(2, 5000, 4, 2, 64, 96, dt, alpha)
            assert bwd(T=5000, dv=96, dtype=dt, da=P[11] if alpha else None, nbytes=n - 1) == mb.EWORKSPACE
            assert n <= mb.memoroid_workspace_bytes(mb.OP_RETENTION_BWD, 2, 5000, 4, 64, 96, 0)
    assert mb.memoroid_scan_retention_workspace_bytes(2, 0, 4, 64, 64, mb.F32) == 0
    assert mb.memoroid_scan_retention_workspace_bytes(2, 10, 4, 60, 64, mb.F32) == 0
    assert mb.memoroid_scan_retention_bwd_workspace_bytes(2, 10, 4, 3, 64, 64, mb.F32, 1) == 0
    assert mb.memoroid_workspace_bytes(mb.OP_RETENTION, -1, 10, 4, 64, 64, 0) == 0


def test_torch_layer_refuses():
    q = torch.zeros(2, 5, 4, 64)
    k = torch.zeros(2, 5, 2, 64)
    a, s = torch.zeros(4), torch.zeros(2, 5, dtype=torch.uint8)
    S = torch.zeros(2, 4, 64, 64)
    bad = [(ValueError, (q[0], k, k, a, s), {}), (ValueError, (q, k[:, :4], k, a, s), {}),
           (ValueError, (q, torch.zeros(2, 5, 3, 64), torch.zeros(2, 5, 3, 64), a, s), {}),
           (ValueError, (q, k[..., :32], k, a, s), {}), (TypeError, (q, k.bfloat16(), k, a, s), {}),
           (TypeError, (q.half(), k.half(), k.half(), a, s), {}), (TypeError, (q, k, k, a[:3], s), {}),
           (TypeError, (q, k, k, a.double(), s), {}), (TypeError, (q, k, k, a, s.bool()), {}),
           (TypeError, (q, k, k, a, s[:, :4]), {}), (TypeError, (q, k, k, a, s), dict(state=S[:1])),
           (TypeError, (q, k, k, a, s), dict(state=S.bfloat16())),
           (ValueError, (q, k, k, a, s), {})]                # the CPU's tensors
    for err, args, kw in bad:
        with pytest.raises(err):
            mb.scan_retention(*args, **kw)
    with pytest.raises(TypeError):
        mb.scan_retention_bwd(q, k, k, a, s, q[:, :4])
    with pytest.raises(TypeError):
        mb.retention_step(q[:, 0], k[:, 0], k[:, 0], a, None)
    with pytest.raises(TypeError):
        mb.retention_step(q[:, 0], k[:, 0], k[:, 0], a, S, s[0])


def rot(q=P[0], k=P[1], pos=P[2], freq=P[3], wq=P[4], wk=P[5], qo=P[6], ko=P[7], eps=1e-6, amp=1.0, inter=0, n=10, H=4, Hk=2,
        d=64, rot=64, dtype=mb.F32):
    return mb.memoroid_rotate_qk(q, k, pos, freq, wq, wk, qo, ko, eps, amp, inter, n, H, Hk, d, rot, dtype, None)


def rotb(q=P[0], k=P[1], pos=P[2], freq=P[3], wq=P[4], wk=P[5], gq=P[6], gk=P[7], dq=P[8], dk_=P[9], dwq=P[10], dwk=P[11],
         eps=1e-6, amp=1.0, inter=0, n=10, H=4, Hk=2, d=64, rot=64, dtype=mb.F32, ws=P[12], nbytes=1 << 40):
    return mb.memoroid_rotate_qk_bwd(q, k, pos, freq, wq, wk, gq, gk, dq, dk_, dwq, dwk, eps, amp, inter, n, H, Hk, d, rot,
                                     dtype, ws, nbytes, None)


@pytest.mark.parametrize("call", [rot, rotb])
def test_rotation_refusals(call):
    nan, inf = float("nan"), float("inf")
    for change in (dict(n=-1), dict(H=-1), dict(Hk=-1), dict(d=-8), dict(rot=-2), dict(rot=3), dict(rot=66), dict(eps=-1.0),
                   dict(eps=nan), dict(eps=inf), dict(amp=nan), dict(amp=inf), dict(pos=None), dict(freq=None),
                   dict(pos=0x900002), dict(freq=0x900002), dict(wq=0x900002), dict(wk=0x900001), dict(q=0x900008),
                   dict(k=0x900008)):
        assert call(**change) == mb.EINVAL, change
    for change in (dict(d=136, rot=0), dict(d=60, rot=0), dict(dtype=mb.C64), dict(dtype=9), dict(H=65536), dict(Hk=65536),
                   dict(n=1 << 50)):
        assert call(**change) == mb.EUNSUPPORTED, change
    for change in (dict(n=0), dict(H=0, Hk=0)):
        assert call(**change) == mb.OK, change
    outs = ("qo", "ko") if call is rot else ("dq", "dk_", "dwq", "dwk")
    ins = ("q", "k", "pos", "freq", "wq", "wk") + (() if call is rot else ("gq", "gk"))
    for o in outs:
        for i in ins + tuple(x for x in outs if x != o):
            assert call(**{o: 0x900000, i: 0x900000}) == mb.EINVAL, (o, i)
    for n in outs[:2] + (("q", "k") if call is rot else ("q", "k", "gq", "gk")):
        assert call(**{n: None}) == mb.EINVAL, n


def test_rotation_gradient_weights_and_workspace():
    assert rotb(wq=None) == mb.EINVAL                       # dwq without wq
    assert rotb(wk=None) == mb.EINVAL
    assert rotb(ws=None) == mb.EWORKSPACE
    need = mb.memoroid_rotate_qk_bwd_workspace_bytes(10, 4, 2, 64, 64, 0, mb.F32)
    assert rotb(nbytes=need - 1) == mb.EWORKSPACE
    assert rotb(ws=0x900008) == mb.EINVAL
    for dt in (mb.F32, mb.BF16):
        for n in (1, 100, 5000, 100000):
            for r in (0, 2, 20, 64):
                for inter in (0, 1):
                    assert mb.memoroid_rotate_qk_bwd_workspace_bytes(n, 4, 2, 64, r, inter, dt) <= \
                        mb.memoroid_workspace_bytes(mb.OP_ROTATE_QK_BWD, 0, n, 4, 2, 64, 0)
    assert mb.memoroid_rotate_qk_bwd_workspace_bytes(10, 4, 2, 60, 20, 0, mb.F32) == 0


def test_rotation_torch_layer_refuses():
    q, k = torch.zeros(2, 5, 4, 64), torch.zeros(2, 5, 2, 64)
    pos, f, w = torch.zeros(2, 5, dtype=torch.int32), torch.ones(32), torch.ones(64)
    for err, args, kw in ((ValueError, (q[0, 0], None, pos, f), {}), (ValueError, (q, k[:1], pos, f), {}),
                          (ValueError, (q, k[..., :32], pos, f), {}), (TypeError, (q, k.bfloat16(), pos, f), {}),
                          (TypeError, (q.half(), k.half(), pos, f), {}), (TypeError, (q, k, pos.long(), f), {}),
                          (TypeError, (q, k, None, f), {}), (TypeError, (q, k, pos[:1], f), {}),
                          (TypeError, (q, k, pos, f.double()), {}), (TypeError, (q, k, pos, torch.ones(33)), {}),
                          (TypeError, (q, k, pos, f), dict(wq=w[:32])), (TypeError, (q, k, pos, f), dict(wk=w.bfloat16())),
                          (ValueError, (q, None, pos, f), dict(wk=w)), (ValueError, (q, k, pos, f), {})):
        with pytest.raises(err):
            mb.rotate_qk(*args, **kw)
    with pytest.raises(TypeError):
        mb.rotate_qk_bwd(q, k, pos, f, q, None)
    for bad in (dict(rot=3), dict(rot=-2), dict(rot=4, base=0.0), dict(rot=4, factor=0.0), dict(rot=4, fast=1.0, slow=2.0)):
        with pytest.raises(ValueError):
            mb.rotary_frequencies(**bad)


def test_rotation_reference_against_differences():
    import rotate_ref
    rng = np.random.default_rng(1)
    for inter in (False, True):
        x, w, g = rng.standard_normal((2, 3, 2, 12)), rng.standard_normal(12), rng.standard_normal((2, 3, 2, 12))
        pos, f = rng.integers(0, 50, (2, 3)), rng.uniform(0, 1, 4)
        args = (pos, f, 1e-3, 1.2, inter)
        _, (dx, _), (dw, _) = rotate_ref.rotate(x, w, *args, grad=g)
        u, uw, h = rng.standard_normal(x.shape), rng.standard_normal(12), 1e-6
        num = ((rotate_ref.rotate(x + h * u, w, *args)[0][0] - rotate_ref.rotate(x - h * u, w, *args)[0][0]) * g).sum() / (2 * h)
        assert abs(num - (dx * u).sum()) <= 1e-6 * (1 + abs(num))
        num = ((rotate_ref.rotate(x, w + h * uw, *args)[0][0] - rotate_ref.rotate(x, w - h * uw, *args)[0][0]) * g).sum() / (2 * h)
        assert abs(num - (dw * uw).sum()) <= 1e-6 * (1 + abs(num))


@pytest.mark.parametrize("call", [scan, bwd])
def test_limits_of_one_launch(call):
    """What no grid or address holds is refused before anything is launched; a
    workspace query of it gives 0."""
    assert call(B=2048, T=1, H=1025, Hk=1025) == mb.EUNSUPPORTED
    assert call(T=1 << 30) == mb.EUNSUPPORTED
    assert call(B=2048, T=1, H=1024, Hk=1024, nbytes=0) == mb.EWORKSPACE
    assert mb.memoroid_scan_retention_workspace_bytes(2048, 1, 1025, 64, 64, mb.F32) == 0
    assert mb.memoroid_scan_retention_bwd_workspace_bytes(2048, 1, 1025, 1, 64, 64, mb.F32, 1) == 0


def test_step_of_one_launch():
    assert step(B=1 << 22, H=1, Hk=1, dv=128) == mb.EUNSUPPORTED
    assert step(B=1 << 24, H=1, Hk=1, dk=8, dv=8) == mb.EUNSUPPORTED


def test_retention_needs_flags():
    x = torch.zeros(1, 3, 2, 8)
    with pytest.raises(TypeError):
        mb.scan_retention(x, x, x, torch.zeros(2), None)


@pytest.mark.parametrize("name", ["q", "k", "v", "alpha", "state"])
def test_step_refuses_inputs_that_want_a_gradient(name):
    """Its result has no graph: a loss on it would miss the step without a word.  Under
    no_grad the call goes on, here to the refusal of the CPU's tensors."""
    x = dict(q=torch.zeros(2, 4, 8), k=torch.zeros(2, 2, 8), v=torch.zeros(2, 2, 8), alpha=torch.zeros(4),
             state=torch.zeros(2, 4, 8, 8))
    x[name].requires_grad_(True)
    with pytest.raises(RuntimeError, match="no gradient"):
        mb.retention_step(**x)
    with torch.no_grad(), pytest.raises(ValueError):
        mb.retention_step(**x)
    with torch.inference_mode(), pytest.raises(ValueError):
        mb.retention_step(**x)


@pytest.mark.parametrize("prepared", [False, True])
def test_workspaces_that_are_not_what_they_count_are_refused(prepared):
    """A view that repeats or skips its memory counts bytes that are not its own to
    write; one on another device is no workspace either.  Refused by both ways that a
    caller's workspace takes, before the library is called."""
    def give(workspace, device):
        if prepared:
            return mb._prepared(lambda: 1024, device, ("diag",), 0, workspace, "memoroid_scan_diag")
        return mb._workspace(1024, device, workspace)

    cpu, other = torch.device("cpu"), torch.device("cuda", 0)
    for bad in (torch.empty(1, dtype=torch.uint8).expand(4096), torch.empty(8192, dtype=torch.uint8)[::2],
                torch.empty(64, 64, dtype=torch.uint8).T[:32]):
        with pytest.raises(ValueError, match="contiguous"):
            give(bad, cpu)
    with pytest.raises(ValueError, match="device"):
        give(torch.empty(4096, dtype=torch.uint8), other)
    if not prepared:
        whole = torch.empty(4096, dtype=torch.uint8)
        assert give(whole, cpu) is whole and give(whole[:10], cpu) is not whole


def test_heads_without_columns_get_as_far_as_the_others():
    """dk = 0 has no default scale of its own; the library refuses it (test_sizes), here
    the layer the CPU's tensors."""
    x, v = torch.zeros(1, 3, 2, 0), torch.zeros(1, 3, 2, 8)
    a, s = torch.zeros(2), torch.zeros(1, 3, dtype=torch.uint8)
    with pytest.raises(ValueError):
        mb.scan_retention(x, x, v, a, s)
    with pytest.raises(ValueError):
        mb.retention_step(x[:, 0], x[:, 0], v[:, 0], a, torch.zeros(1, 2, 0, 8))
