"""Layer norm where values come near the ends of fp32's range, and past 2^31 elements."""
import pytest

import gated_ref as ref
from conftest import announce, cond_err
from test_gpu_norm import DEV, DT, E, np64

torch = pytest.importorskip("torch")
from paper_2402_09900_amd import binding as mb  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [3, 64, 250, 2048, 5000, 16384])
@pytest.mark.parametrize("size", [1e37, 3e38, -2.5e38])
def test_rows_whose_sum_is_past_the_range(dtype, d, size):
    """Large values of one sign: their sum is no float, their mean is.  Where the deviations
    are large too the row is the bias, where there are none it is the bias to the rounding of
    the mean; no gradient comes through either but the one of s."""
    announce("norm sums past the range %s d=%d size=%g" % (dtype, d, size))
    x = torch.full((5, d), size, device=DEV)
    x[1, ::2] *= 0.5
    x[2, 0] *= 0.75
    x[3, -1] = 0.0
    x[4] = torch.randn(d, device=DEV)
    x = x.to(DT[dtype])
    w, b = torch.rand(d, device=DEV) + 0.5, torch.randn(d, device=DEV)
    y, st = mb.norm_rows(x, w, b, keep_stats=True)
    want = x.double().mean(-1)
    # half a step for every add of a lane and across lanes and wavefronts, 40 at most
    assert bool(((st[:4, 0].double() - want[:4]).abs() <= 40 * 2.0 ** -24 * x[:4].double().abs().mean(-1)).all())
    for row in (1, 2, 3):
        assert float(st[row, 1]) == 0.0 and torch.equal(y[row], b.to(y.dtype)), row
    assert bool(torch.isfinite(y).all())
    assert torch.equal(y[4], mb.norm_rows(x[4:], w, b)[0])
    gy, gs = torch.randn_like(x), torch.randn_like(x)
    dx, dres, dw, db = mb.norm_rows_bwd(x, st, gy, w, torch.zeros_like(x), gs)
    assert torch.equal(dx[1:4], gs[1:4]) and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())


def test_weights_past_32_bits():
    """More than 2^31 elements of which the last 64 rows are not zero: the gradients of weight
    and bias against those rows' in 64 bits (144 E: test_gpu_norm.py)."""
    announce("norm weights past 2^31 elements")
    n, d, m = 1050000, 2048, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, gy = (torch.zeros(n, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t in (x, gy):
        t[-m:] = torch.randn(m, d, device=DEV, generator=g).to(torch.bfloat16)
    w = torch.rand(d, device=DEV, generator=g)
    _, st = mb.norm_rows(x, w, keep_stats=True)
    _, _, dw, db = mb.norm_rows_bwd(x, st, gy, w)
    _, gw, gb = ref.norm_grads(np64(x[-m:]), np64(w), 1e-5, np64(gy[-m:]))
    assert cond_err(np64(dw), *gw) <= 144 * E
    assert cond_err(np64(db), *gb) <= 144 * E
