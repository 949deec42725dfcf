"""The torch layer of the gated recurrence, layer norm and dropout under torch's other
ways of calling: what it cannot answer it refuses, before it looks where tensors lie, so
that the refusals are tested here on the CPU."""
import pytest

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
