"""Layer norm and its gradients at deviations and offsets near the ends of fp32's range, where the definition's values
are finite.  Reference and bars are those of test_layer_norm_gpu, with what the small deviations' own squares lose."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_19509_amd import gcx  # noqa: E402
from test_layer_norm_gpu import everything, problem, reference  # noqa: E402

pytestmark = pytest.mark.gpu
WIDTHS = [5, 60, 64, 1003, 4096, 10003, 16384, 16390, 20001, 40001]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_tiny_deviations_without_eps(d, dtype):
    """Deviations of 2^-65 or so: rstd is 2^65, and its square no float.  Squares of deviations are multiples of 2^-149,
    each off by 2^-150 at most, as is their mean: 2^-149 rstd^2 of it (2^-19 for a row of 2^-65), so half of that of
    rstd and of h."""
    x, dy, gamma, beta = problem(2, 5, d, dtype)
    x = x * 2.0 ** -65
    ref, bar = reference(x, dy, gamma, beta, 0.0)
    assert float(ref["rstd"].max()) > 2.0 ** 64.1
    h = ((x.double() - ref["mean"][..., None]) * ref["rstd"][..., None]).abs()
    a = (dy.double() * gamma.double()).abs()
    rel = 2.0 ** -150 * ref["rstd"].square()[..., None]
    more = {"mean": 0.0, "rstd": rel[..., 0] * ref["rstd"], "y": rel * h * gamma.double().abs(),
            "dx": rel * ref["rstd"][..., None] * (a + a.mean(-1, keepdim=True) + 3 * h * (a * h).mean(-1, keepdim=True)),
            "dgamma": (rel * dy.double().abs() * h).sum(1), "dbeta": 0.0}
    for k, v in everything(x, dy, gamma, beta, eps=0.0).items():
        b = bar[k] + more[k] + (2.0 ** -8 * ref[k].abs() * 1.01 if dtype == torch.bfloat16 and k in ("y", "dx") else 0.0)
        off = (v.double() - ref[k]).abs()
        assert bool((off <= b).all()), (k, float((off / b).max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("level", [2.0 ** 108, -2.0 ** 108])
@pytest.mark.parametrize("d", WIDTHS + [1, 2, 7, 513, 2051, 8196, 32765])
def test_constant_rows_far_off_zero(d, level, dtype):
    """Every sum of a row of 2^108 is exact, so h = 0 and dx = rstd (a - mean a) to the roundings of sums of d terms; what
    a kernel makes of the places past a row's end (of zeros there: h = -2^128) is not among them."""
    _, dy, gamma, beta = problem(2, 5, d, dtype)
    x = torch.full_like(dy, level)
    x[1, 1:3] = 0.0
    got = everything(x, dy, gamma, beta, eps=2.0 ** -40)
    assert torch.equal(got["mean"].double(), x[..., 0].double()) and bool((got["rstd"] == 2.0 ** 20).all())
    assert torch.equal(got["y"], beta.to(dtype).expand_as(x)) and not got["dgamma"].any()
    a = dy.double() * gamma.double()
    want = 2.0 ** 20 * (a - a.mean(-1, keepdim=True))
    bar = 2.0 ** 20 * (2 * d ** 0.5 + 8) * 2.0 ** -24 * (a.abs() + a.abs().mean(-1, keepdim=True))
    if dtype == torch.bfloat16:
        bar = bar + 2.0 ** -8 * (want.abs() + bar)
    assert bool(((got["dx"].double() - want).abs() <= bar).all())
    n = dy.shape[1]
    assert bool(((got["dbeta"].double() - dy.double().sum(1)).abs() <= (2 * n ** 0.5 + 8) * 2.0 ** -24 * dy.double().abs().sum(1)).all())
