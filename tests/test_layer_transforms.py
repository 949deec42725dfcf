"""The torch layer of the gated recurrence, layer norm and dropout under torch's other
ways of calling: what it cannot answer it refuses, before it looks where tensors lie, so
that the refusals are tested here on the CPU."""
import pytest

from conftest import announce

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fwd  # noqa: E402
from paper_2402_09900_amd import binding as mb  # noqa: E402

X, GATES, ALPHA = torch.zeros(2, 5, 8), torch.zeros(2, 5, 2, 8), torch.zeros(8)
START, STATE, RNG = torch.zeros(2, 5, dtype=torch.uint8), torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
ROW, ROW_GATES = torch.zeros(2, 8), torch.zeros(2, 2, 8)

# name: the call, the inputs that a gradient may hang on
DIFFERENTIABLE = {
    "gated_scan": (lambda **k: mb.gated_scan(start=START, **k), dict(x=X, gates=GATES, alpha=ALPHA, state=STATE)),
    "layer_norm": (mb.layer_norm, dict(x=X, weight=ALPHA, bias=ALPHA, residual=X)),
    "layer_norm_p": (lambda **k: mb.layer_norm(p=0.5, rng=RNG, **k), dict(x=X, residual=X)),
    "dropout": (lambda **k: mb.dropout(p=0.5, rng=RNG, **k), dict(x=X, residual=X)),
    "gated_step": (mb.gated_step, dict(x=ROW, gates=ROW_GATES, alpha=ALPHA, state=STATE)),
}


def each_input(calls):
    return [(name, k) for name, (_, inputs) in calls.items() for k in inputs]


@pytest.mark.parametrize("name,which", each_input(DIFFERENTIABLE))
@pytest.mark.parametrize("grad", [False, True])
def test_forward_mode_is_refused(name, which, grad):
    """A tangent that nobody would carry on is refused, under no_grad too (which leaves
    forward mode on); where forward mode is off, a dual tensor is its primal."""
    f, inputs = DIFFERENTIABLE[name]
    with fwd.dual_level(), torch.set_grad_enabled(grad):
        k = {n: t.clone() for n, t in inputs.items()}
        k[which] = fwd.make_dual(k[which], torch.ones_like(k[which]))
        with pytest.raises(RuntimeError, match="forward mode"):
            f(**k)
        with fwd._set_fwd_grad_enabled(False), pytest.raises(ValueError, match="CUDA"):
            f(**k)


@pytest.mark.parametrize("name", DIFFERENTIABLE)
def test_functional_jvp_is_refused(name):
    f, inputs = DIFFERENTIABLE[name]
    with pytest.raises(RuntimeError, match="forward mode"):
        torch.func.jvp(lambda x: f(**{**inputs, "x": x}), (inputs["x"],), (torch.ones_like(inputs["x"]),))


# ------------------------------------------------------------------ recording

STATS, KEPT = torch.zeros(2, 5, 2), torch.zeros(2, 1, 8)
RAW = {
    "scan_gated": lambda x: mb.scan_gated(x, GATES, ALPHA, START),
    "scan_gated_bwd": lambda x: mb.scan_gated_bwd(x, GATES, ALPHA, START, KEPT, x),
    "norm_rows": lambda x: mb.norm_rows(x, ALPHA),
    "norm_rows_bwd": lambda x: mb.norm_rows_bwd(x, STATS, x, ALPHA),
    "drop_rows": lambda x: mb.drop_rows(x, 0.5, RNG),
}


def of_x(name):
    f, inputs = DIFFERENTIABLE[name]
    return lambda x: f(**{**inputs, "x": x})


def input_of(name):
    return ROW if name == "gated_step" else X


FORMS = {**RAW, **{name: of_x(name) for name in DIFFERENTIABLE}}


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("grad", [False, True])
def test_traces_are_refused(name, grad):
    """A trace would hold the new memory of the results and not the call that fills it."""
    x = input_of(name).clone().requires_grad_(grad and name != "gated_step")
    with pytest.raises(RuntimeError, match="cannot be traced"):
        torch.jit.trace(FORMS[name], (x,))
    with pytest.raises(ValueError, match="CUDA"):                    # (and again afterwards as before)
        FORMS[name](x)


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("mode", ["real", "fake", "symbolic"])
def test_graphs_of_operators_are_refused(name, mode):
    from torch.fx.experimental.proxy_tensor import make_fx

    with pytest.raises(RuntimeError, match="cannot be traced"):
        make_fx(FORMS[name], tracing_mode=mode)(input_of(name))


@pytest.mark.parametrize("name", FORMS)
def test_fake_tensors_are_refused(name):
    from torch._subclasses.fake_tensor import FakeTensorMode

    with FakeTensorMode(allow_non_fake_inputs=True) as mode:
        x = mode.from_tensor(input_of(name))
        with pytest.raises(RuntimeError, match="cannot be traced"):
            FORMS[name](x)


def test_other_modes_are_let_through():
    """A dispatch mode that only looks on (a count of operations, checkpointing) does not
    stand in the way."""
    from torch.utils.flop_counter import FlopCounterMode

    with FlopCounterMode(display=False), pytest.raises(ValueError, match="CUDA"):
        mb.layer_norm(X)


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("through", [torch.func.vmap, lambda f: torch.func.grad(lambda x: f(x).sum()), torch.func.functionalize])
def test_transforms_are_refused(name, through):
    x = input_of(name)
    if through is torch.func.vmap:
        x = torch.stack([x, x])
    with pytest.raises((RuntimeError, ValueError)):
        through(FORMS[name])(x)


@pytest.mark.gpu
def test_graph_of_a_backward_pass_is_refused():
    """A graph of operators that begins behind the forward call; afterwards the same pass
    gives the gradient."""
    from torch.fx.experimental.proxy_tensor import make_fx

    announce("transforms: backward pass in a graph of operators")
    dev = "cuda:0"
    x = torch.randn(2, 5, 8, device=dev, requires_grad=True)
    gates, alpha, start, rng = GATES.to(dev), ALPHA.to(dev) + 0.5, START.to(dev), RNG.to(dev)
    for y in (mb.gated_scan(x, gates, alpha, start), mb.layer_norm(x), mb.dropout(x, 0.5, rng)):
        def back(g, y=y):
            return torch.autograd.grad(y, x, g, retain_graph=True)[0]

        up = torch.randn_like(y)
        want = back(up)
        with pytest.raises(RuntimeError, match="cannot be traced"):
            make_fx(lambda g: back(g))(up)
        assert torch.equal(back(up), want)


@pytest.mark.gpu
@pytest.mark.parametrize("through", ["vmap", "grad", "functionalize"])
def test_tensors_without_memory_are_refused(through):
    """On the device, where nothing else is wrong with them, an optional input too: it would
    count as not given."""
    announce("transforms: no memory in %s" % through)
    dev = "cuda:0"
    x, row, alpha = X.to(dev), ROW.to(dev), ALPHA.to(dev)
    gates, row_gates, start, state = GATES.to(dev), ROW_GATES.to(dev), START.to(dev), STATE.to(dev)
    wrap = dict(vmap=lambda f: lambda t: torch.func.vmap(f)(torch.stack([t, t])),
                grad=lambda f: torch.func.grad(lambda t: f(t).sum()), functionalize=torch.func.functionalize)[through]
    calls = [(mb.layer_norm, x), (lambda r: mb.layer_norm(x, residual=r)[0], x), (lambda w: mb.layer_norm(x, w), alpha),
             (lambda w: mb.layer_norm(x, None, w), alpha), (lambda r: mb.norm_rows(x, residual=r)[0], x),
             (lambda t: mb.dropout(t, 0.0, None), x), (lambda r: mb.dropout(x, 0.0, None, residual=r), x),
             (lambda r: mb.drop_rows(x, 0.0, None, residual=r), x), (lambda t: mb.gated_scan(t, gates, alpha, start), x),
             (lambda s: mb.gated_scan(x, gates, alpha, start, s), state), (lambda s: mb.scan_gated(x, gates, alpha, start, s), state),
             (lambda t: mb.gated_step(t, row_gates, alpha, state), row)]
    for n, (f, t) in enumerate(calls):
        with pytest.raises((RuntimeError, ValueError)):
            wrap(f)(t)
            assert False, "call %d went through" % n


@pytest.mark.gpu
def test_onlookers_see_the_same_results():
    """Dispatch modes that only look on, a level of forward mode that no input belongs to,
    and both kinds of checkpointing: the results and gradients of a plain call."""
    from torch.utils._python_dispatch import TorchDispatchMode
    from torch.utils.checkpoint import CheckpointPolicy, checkpoint, create_selective_checkpoint_contexts
    from torch.utils.flop_counter import FlopCounterMode

    class Looks(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    announce("transforms: onlookers")
    dev = "cuda:0"
    torch.manual_seed(0)
    x, res = (torch.randn(2, 300, 8, device=dev) for _ in range(2))
    gates, alpha = torch.randn(2, 300, 2, 8, device=dev), torch.rand(8, device=dev)
    start, rng = torch.zeros(2, 300, dtype=torch.uint8, device=dev), RNG.to(dev)
    up = torch.randn_like(x)
    leaves = [t.requires_grad_(True) for t in (x, res, gates, alpha)]

    def block(x, res, gates, alpha):
        y, s = mb.layer_norm(x, alpha, residual=res, p=0.1, rng=rng)
        return mb.dropout(mb.gated_scan(y, gates, alpha, start), 0.2, rng, 1, s)

    def both(f=block):
        y = f(*leaves)
        y.backward(up)
        got = (y.detach(), *[t.grad for t in leaves])
        for t in leaves:
            t.grad = None
        return got

    want = both()

    def policy(ctx, op, *args, **kwargs):
        return CheckpointPolicy.MUST_SAVE

    def same(got):
        return all(torch.equal(a, b) for a, b in zip(got, want))

    with FlopCounterMode(display=False):
        assert same(both())
    with Looks():
        assert same(both())
    with fwd.dual_level():
        assert same(both())
    assert same(both(lambda *a: checkpoint(block, *a, use_reentrant=False)))
    assert same(both(lambda *a: checkpoint(block, *a, use_reentrant=True)))
    assert same(both(lambda *a: checkpoint(block, *a, use_reentrant=False,
                                           context_fn=lambda: create_selective_checkpoint_contexts(policy))))
