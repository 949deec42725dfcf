"""Gradients of the torch layer's autograd forms have no derivative: wherever a second one
would be asked for, the backward pass raises, and none is left out without a word."""
import pytest

from conftest import announce

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def forms():
    g = torch.Generator(device=DEV)
    g.manual_seed(3)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    start = torch.zeros(2, 9, dtype=torch.uint8, device=DEV)
    rng = torch.tensor([7, 1], dtype=torch.int64, device=DEV)
    x, gates, alpha, state = normal(2, 9, 16), normal(2, 9, 2, 16), torch.rand(16, device=DEV, generator=g) + 0.1, normal(2, 16)
    res, w, b = normal(2, 9, 16), normal(16), normal(16)
    return {
        "gated": (lambda x, gates, alpha, state: mb.gated_scan(x, gates, alpha, start, state, final_state=True), (x, gates, alpha, state)),
        "norm": (lambda x, w, b, res: mb.layer_norm(x, w, b, residual=res), (x, w, b, res)),
        "norm_p": (lambda x, w, b, res: mb.layer_norm(x, w, b, residual=res, p=0.3, rng=rng), (x, w, b, res)),
        "norm_alone": (lambda x, b: (mb.layer_norm(x, None, b),), (x, b)),
        "dropout": (lambda x: (mb.dropout(x, 0.3, rng),), (x,)),
    }


@pytest.mark.parametrize("name", ["gated", "norm", "norm_p", "norm_alone", "dropout"])
def test_no_second_derivative_is_left_out(name):
    announce("twice %s" % name)
    f, inputs = forms()[name]
    torch.manual_seed(0)
    ups = [torch.randn_like(y) for y in f(*inputs)]
    for j in range(len(inputs)):
        leaves = [t.clone().requires_grad_(k == j) for k, t in enumerate(inputs)]
        x = leaves[j]

        def loss():
            return sum((y * y * u).sum() for y, u in zip(f(*leaves), ups))

        first, = torch.autograd.grad(loss(), x)
        g, = torch.autograd.grad(loss(), x, create_graph=True)
        assert torch.equal(g, first) and g.requires_grad
        # the gradient in the middle of a sum, whose other part needs no second derivative
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.grad(loss() + g.square().sum(), x)
        # with respect to what came from behind
        up = [u.clone().requires_grad_(True) for u in ups]
        g, = torch.autograd.grad(f(*leaves), x, up, create_graph=True)
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.grad(g.sum(), up[0])
        # with respect to another input
        both = [t.clone().requires_grad_(True) for t in inputs]
        out = f(*both)
        g, = torch.autograd.grad(out, both[j], ups, create_graph=True)
        for t in both:
            with pytest.raises(RuntimeError, match="twice"):
                torch.autograd.grad(g.sum(), t, retain_graph=True)
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.functional.jvp(lambda t: f(*[t if k == j else v for k, v in enumerate(inputs)])[0], inputs[j],
                                          torch.ones_like(inputs[j]))


def test_gradients_that_go_through_unchanged():
    """The residual's gradient is the one that came, and x's without dropout: they have the
    derivatives of an identity."""
    announce("twice: identities")
    rng = torch.tensor([7, 1], dtype=torch.int64, device=DEV)
    x, r = (torch.randn(5, 16, device=DEV, requires_grad=True) for _ in range(2))
    up = torch.randn(5, 16, device=DEV, requires_grad=True)
    for p, leaf in ((0.3, r), (0.0, r), (0.0, x)):
        g, = torch.autograd.grad(mb.dropout(x, p, rng, residual=r), leaf, up, create_graph=True)
        assert torch.equal(g, up)
        gg, = torch.autograd.grad((g * g).sum(), up)
        assert torch.equal(gg, 2 * up)


@pytest.mark.filterwarnings("ignore:Using backward")
def test_gradients_in_a_graph_are_used_once():
    """create_graph as such changes nothing: the same gradients, also for one leaf in two
    places, and they can be accumulated and cleared."""
    announce("twice: create_graph")
    x = torch.randn(5, 16, device=DEV, requires_grad=True)
    for _ in range(2):
        y, s = mb.layer_norm(x, residual=x)
        ones = (torch.ones_like(y), torch.ones_like(s))
        want, = torch.autograd.grad((y, s), x, ones, retain_graph=True)
        torch.autograd.backward((y, s), ones, create_graph=True)
        assert torch.equal(x.grad, want)
        x.grad = None
